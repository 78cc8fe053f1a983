"""Source rules and host logic of the ranked cache and shared prefix kernels (no GPU)."""
import os
import re

import pytest

import paper_2603_19664_b200 as kvd

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_19664_b200", "csrc")
KERNELS = {}
for _f in ("kvd_prefill_weights.cu", "kvd_shared_prefix.cu", "kvd_evict.cu", "kvd_attention.cu"):
    _text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, _f)).read())
    for _m in re.finditer(r"__global__ void[^;{]*?(kvd_\w+)\(([^{]*)\) \{", _text):
        depth, i = 1, _m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(_text[i], 0)
            i += 1
        KERNELS[_m.group(1)] = (_m.group(2), _text[_m.end():i])
NEW = ["kvd_prefill_weights_kernel", "kvd_prefill_weights_sum_kernel", "kvd_shared_prefix_kernel", "kvd_evict_select_kernel",
       "kvd_evict_rows_kernel", "kvd_shared_merge_kernel", "kvd_attn_merge_weigh_kernel"]


@pytest.mark.parametrize("name", NEW)
def test_nothing_of_the_predecessor_is_read_before_the_wait(name):
    args, body = KERNELS[name]
    assert "__restrict__" not in args and "__ldg" not in body and body.count("grid_dependency_wait();") == 1
    assert not re.search(r"P\.(q|q_pos|k|v|weights|positions|part_o|part_ml|ml|cols|neg_lse|in|out)\b", body[:body.index("grid_dependency_wait();")])


@pytest.mark.parametrize("name", [n for n in NEW if "tmem_claim" in KERNELS[n][1]])
def test_dependents_start_only_after_tensor_memory_is_allocated(name):
    """The allocation waits without a limit: a dependent let in first could hold the columns it waits for."""
    body = KERNELS[name][1]
    claim, start = body.index("tmem_claim"), body.index("grid_launch_dependents")
    assert claim < start and "__syncthreads()" in body[claim:start]
    # ... and is given back behind a barrier that every role reaches, whatever ran out of time
    rest = body[start:body.index("tmem_dealloc")]
    for m in reversed(list(re.finditer(r"\[&\]\([^)]*\) \{", rest))):  # (what lambdas return)
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(rest[i], 0)
            i += 1
        rest = rest[:m.start()] + rest[i:]
    assert "return" not in rest


def test_every_wait_has_a_limit():
    for f in ("kvd_prefill_weights.cu", "kvd_shared_prefix.cu"):
        text = open(os.path.join(CSRC, f)).read()
        for m in re.finditer(r"while \(!mbar_try_wait[^)]*\)[^{;]*[{;]?", text):
            assert "tmo" in text[m.start():m.end() + 300] or "timeout_ns" in text[m.start():m.end() + 300]


def test_scratch_sizes():
    d = kvd.make_desc(1, 64, 32, 8, 128, 1e-6, False, 1e-6, max_tokens_per_seq=65536, max_batch=64)
    assert kvd.kvd_weights_scratch_bytes(d, 0, 10) == kvd.kvd_weights_scratch_bytes(d, 1, 0) == 0
    one = kvd.kvd_weights_scratch_bytes(d, 1, 5000)
    n, chunk = kvd.kvd_attention_split(128, 8, 63, 5062)
    assert one >= 32 * 4 * n * chunk  # whole chunks over the span, wherever it begins
    assert kvd.kvd_weights_scratch_bytes(d, 200, 5000) == kvd.kvd_weights_scratch_bytes(d, 64, 5000)  # a launch's sequences
    assert kvd.kvd_prefill_weights_scratch_bytes(d, 0, 5) == kvd.kvd_prefill_weights_scratch_bytes(d, 5, 0) == 0
    assert kvd.kvd_prefill_weights_scratch_bytes(d, 5, 2**30 + 1) == 0
    for rows in (1, 64, 4096, 65536):  # far from a matrix of scores
        assert 0 < kvd.kvd_prefill_weights_scratch_bytes(d, rows, 32768) < 600 << 20
    bad = kvd.make_desc(1, 64, 7, 4, 128, 1e-6, False, 1e-6)
    assert kvd.kvd_weights_scratch_bytes(bad, 1, 5) == kvd.kvd_prefill_weights_scratch_bytes(bad, 1, 5) == 0
