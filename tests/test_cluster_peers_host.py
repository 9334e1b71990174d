"""Kernels whose CTAs reach into each other's shared memory, read as text: a CTA of a cluster touches a
peer's memory only after a cluster barrier that every CTA has arrived at, since before that the peer may
not have started; and none ends between its arrival and its wait."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2604_10044_gb300", "csrc")
PEER = r"\bmap_shared_rank\(|\bmapa\.shared::cluster|\bpeer_addr\("
MET = r"\bcl\.sync\(\)|\bpeers_wait\(\)|\bcluster_wait\(\)|barrier\.cluster\.wait"


def _kernels(name):
    """(name, body) of the kernels of a file that reach into a peer's memory"""
    src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    out = []
    for m in re.finditer(r"__global__ void[^;{]*?(\w+)\((?:[^()]|\([^()]*\))*\)\s*\{", src):
        at, depth = m.end(), 1
        while depth:
            depth += {"{": 1, "}": -1}.get(src[at], 0)
            at += 1
        if re.search(PEER, src[m.end():at]):
            out.append((m.group(1), src[m.end():at]))
    return out


@pytest.mark.parametrize("name,kernels", [("lg_verify.cu", {"verify_pick_kernel"}),
                                          ("lg_q4_attend.cu", {"q4_attend_kernel"}),
                                          ("lg_pick.cu", {"pick_token_kernel"})])
def test_peers_have_started_before_they_are_reached(name, kernels):
    found = _kernels(name)
    assert {k for k, _ in found} == kernels
    for kernel, body in found:
        met = re.search(MET, body)
        assert met and met.start() < re.search(PEER, body).start(), kernel


def test_verification_waits_for_whom_it_arrived():
    """the arrival comes first, so that the barrier's way is behind the joining of rows; between it and
    the first wait on the common path every return has a wait of its own"""
    body = dict(_kernels("lg_verify.cu"))["verify_pick_kernel"]
    arrive = body.index("peers_arrive();")
    assert arrive < body.index("pdl_enter();") and body.count("peers_arrive();") == 1
    waits = [m.start() for m in re.finditer(r"peers_wait\(\);", body)]
    assert len(waits) == 2 and waits[-1] < re.search(PEER, body).start()
    returns = [m.start() for m in re.finditer(r"\breturn;", body[:waits[-1]])]
    assert len(returns) == 1 and waits[0] < returns[0]
    assert not body[waits[0] + len("peers_wait();"):returns[0]].strip()
