"""Source rules of kernels that give up a wait: what is on its way into a CTA's shared memory arrives before the CTA ends.  (A wait runs out when
something else is broken; no run shows reliably what a late copy would write over.)"""
import re

from test_launch_rules import KERNELS, TEXT


def test_copies_of_the_cache_are_waited_for_whatever_the_abort_flag_says():
    text, body = TEXT["kvd_cache4.cu"], KERNELS["kvd_cache4_attention_kernel"][1]
    given_up = text[text.index("void c4_give_up("):text.index("c4_large(")]
    behind = given_up[given_up.index("raise(P.status, STATUS_TIMEOUT, abort_flag);"):]
    # not the flag that was just raised, but one that nobody raises; the limit stays
    assert re.findall(r"warp_wait\(([^;]*)\);", behind) == ["W.bars + 8 * (F.attended % S), (F.attended / S) & 1, never, P.timeout_ns, lane"]
    assert re.findall(r"s_never\s*=[^;]*;", body) == ["s_never = 0;"] and not re.search(r"\*never\s*=", text)
    # all parts that may be on their way: as many as the ring has stages
    assert "for (int j = F.i / TP * TP; j < min(F.end, F.i / TP * TP + S * TP); j += TP, ++F.attended)" in given_up
    # every wait for a copy that runs out goes there, with both flags
    waits = [m.end() for m in re.finditer(r"!warp_wait\([^;{]*\{", text)]
    assert len(waits) == 2 and all(text[at:].lstrip().startswith("c4_give_up<DH>(") for at in waits)
    assert text.count("STATUS_TIMEOUT") == 1
    assert "&s_abort, &s_never, F)" in body and re.search(r"c4_large<DH, QB>\([^;]*&s_abort, &s_never", body) and re.search(r"C4Large<DH, QB> L\{[^;]*&s_abort, &s_never", body)


def test_a_cta_of_a_cluster_keeps_its_memory_for_the_others():
    body = KERNELS["kvd_sample_kernel"][1]
    assert re.search(r"auto leave = \[&\]\(\) \{\s*if \(s_abort != 0\) cluster_stay\(\);\s*\};", body)
    # behind the last wait every way out goes by it (the way out before is that of a row without a message, behind a barrier of all)
    behind = body[body.index("heard(SM_SHARES);"):]
    ways = len(re.findall(r"\breturn;", behind)) + 1
    assert len(re.findall(r"leave\(\);\s*(?:return;|\}\s*$)", behind)) == ways == 3
    before = body[:body.index("heard(SM_SUMS);")]
    assert re.search(r"cluster_wait\(\);\s*return;", before)
