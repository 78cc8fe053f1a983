"""Source rules of kernels that give up a wait: what is on its way into a CTA's shared memory arrives before the CTA ends.  (A wait runs out when
something else is broken; no run shows reliably what a late copy would write over.)"""
import re

from test_launch_rules import KERNELS


def test_copies_of_the_cache_are_waited_for_whatever_the_abort_flag_says():
    body = KERNELS["kvd_cache4_attention_kernel"][1]
    given_up = body[body.index("raise(P.status, STATUS_TIMEOUT"):]
    given_up = given_up[:given_up.index("return;")]
    waits = re.findall(r"warp_wait\(([^;]*)\);", given_up)
    assert waits
    for w in waits:  # not the flag that was just raised, but one that nobody raises; the limit stays
        assert "&s_never" in w and "s_abort" not in w and "P.timeout_ns" in w
    assert re.findall(r"s_never\s*=[^;]*;", body) == ["s_never = 0;"] and body.count("s_never") == 2 + len(waits)
    # all parts that may be on their way: as many as the ring has stages
    assert re.search(r"for \(int j = i / TP \* TP; j < min\(end, i / TP \* TP \+ S \* TP\); j \+= TP, \+\+attended\)", given_up)


def test_a_cta_of_a_cluster_keeps_its_memory_for_the_others():
    body = KERNELS["kvd_sample_kernel"][1]
    assert re.search(r"auto leave = \[&\]\(\) \{\s*if \(s_abort != 0\) cluster_stay\(\);\s*\};", body)
    # behind the last wait every way out goes by it (the way out before is that of a row without a message, behind a barrier of all)
    behind = body[body.index("heard(SM_SHARES);"):]
    ways = len(re.findall(r"\breturn;", behind)) + 1
    assert len(re.findall(r"leave\(\);\s*(?:return;|\}\s*$)", behind)) == ways == 3
    before = body[:body.index("heard(SM_SUMS);")]
    assert re.search(r"cluster_wait\(\);\s*return;", before)
