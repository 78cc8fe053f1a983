"""What the sources of the ranked cache have to hold for races and sizes that no run shows (no GPU)."""
import os
import re

import pytest

from test_ranked_cache_rules import CSRC, KERNELS


def _block(text, at):
    """The text of the brace block that opens at or after `at`."""
    at = text.index("{", at)
    depth, i = 1, at + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        i += 1
    return text[at:i]


def test_no_weight_is_read_once_a_cta_of_the_cluster_may_write_it():
    """In the one-launch form every CTA of a cluster reads all of a sequence's weights and the first one writes them back, in
    place to where others read: behind the last read that all of them make there is a barrier of the cluster."""
    body = KERNELS["kvd_evict_select_kernel"][1]
    barrier = "if (copies > 1) cluster_sync_all();"
    write = body.index("P.weights_out[")
    reads = [m.start() for m in re.finditer(r"\bw\[slot0 \+ i\]", body) if "copy == 0" not in body[body.rindex("\n", 0, m.start()):m.start()]]
    assert len(reads) == 2 and max(reads) < write
    again = _block(body, body.index("if (T == EV_PROTECTED)"))
    for text in (body[:body.index("if (T == EV_PROTECTED)")], again):
        read = max(m.end() for m in re.finditer(r"\bw\[slot0 \+ i\]", text))
        assert barrier in text[read:]
    # (a barrier that only some CTAs reached would hang: the branch hangs on T alone, which all of them find from the same keys)
    assert "rank" not in again and "copy " not in again


def test_the_selections_lists_fit_the_counts_they_follow():
    """A single CTA's holes (half of its slots at most) lie where its counts were, a small cache's places behind them where the
    cluster's were: a size that breaks either does not compile."""
    text = open(os.path.join(CSRC, "kvd_evict.cu")).read()
    struct = _block(text, text.index("struct EvictShared"))
    assert "hist[3][EV_BINS];" in struct and "sum[3][EV_BINS];" in struct and struct.index("hist[3]") < struct.index("sum[3]")
    body = KERNELS["kvd_evict_select_kernel"][1]
    assert re.search(r"\*holes = &S\.hist\[0\]\[0\], \*source = &S\.sum\[0\]\[0\]", body)
    consts = {m.group(1): int(eval(m.group(2))) for m in re.finditer(r"constexpr int (EV_\w+) = ([0-9 <]+);", text)}
    claims = re.findall(r"static_assert\(([^\"]*), \"", text)

    def compiles(**changed):
        return all(eval(c, {}, {**consts, **changed}) for c in claims)

    words = 3 * consts["EV_BINS"]
    assert compiles() and compiles(EV_RUN=2 * words) and compiles(EV_SMALL=words)
    assert not compiles(EV_RUN=2 * words + 2) and not compiles(EV_SMALL=words + 1)


@pytest.mark.parametrize("kernel,accesses", [
    ("kvd_prefill_weights_kernel", [r"P\.ml\[at\]", r"__ldcg\(src \+", r"s_sum\[grp\]\[[^;]*\] \+=", r"\bdst\[i\] = ", r"\bs_tile\[i\] = "]),
    ("kvd_prefill_weights_sum_kernel", [r"__ldcg\(P\.cols \+"]),
])
def test_the_checking_build_tests_what_the_prompt_weights_kernels_index(kernel, accesses):
    """Row tiles, statistics, sums in shared memory and partial columns: every index derived on the device stands behind a test."""
    body = KERNELS[kernel][1]
    for access in accesses:
        found = list(re.finditer(access, body))
        assert found, access
        for m in found:  # in the access's line, or in the few ahead of it
            lines = body[:m.start()].split("\n")[-6:]
            assert any("KVD_BOUNDS_OK(" in line for line in lines), body[m.start():m.end()]
    # every such access is one of those
    assert not re.search(r"P\.ml\[\(|P\.cols\[", body)
