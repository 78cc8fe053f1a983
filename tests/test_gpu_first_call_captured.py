"""The very first call of a process, of every operator over a 4-bit cache and of sampling, may be one that is captured into a graph."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu

PROGRAM = """
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import torch
import paper_2603_19664_b200 as kvd
from test_gpu_cache4 import DT, SHAPES, Cache, ints, open_ctx, rows
shape, dtype, what = {shape!r}, {dtype}, {what!r}
ctx, desc = open_ctx(shape, dtype)
nq, nkv, dh = SHAPES[shape]
c = Cache(desc, [70, 3], spare=9)
k, q = rows(1, 73, nkv, dh, dtype), rows(2, 2, nq, dh, dtype)
out, ko, first, zero = torch.zeros_like(q), torch.zeros_like(k), ints(0, 0), ints(0, 0)
scratch = torch.empty(max(kvd.kvd_cache4_scratch_bytes(desc, 2), kvd.kvd_pages_scratch_bytes(c.pages)), dtype=torch.uint8, device="cuda")
x, u, t = rows(3, 20, 1, 5000, dtype).view(20, 5000), torch.full((20,), 0.5, device="cuda"), ints(*[-1] * 20)
calls = dict(append=lambda: ctx.kvd_cache4_append(0, c.tuple, [0, 1], [70, 3], zero, k, k, nkv * dh),
             expand=lambda: ctx.kvd_cache4_expand(0, c.tuple, [0, 1], [70, 3], zero, ko, ko.clone(), nkv * dh),
             attend=lambda: ctx.kvd_decode_attention_cache4(0, c.tuple, [0, 1], q, 0, 0.0, out, scratch),
             grow=lambda: ctx.kvd_pages_grow(c.tuple, [0, 1], [1, 1], first),
             fork=lambda: ctx.kvd_pages_fork(c.tuple, [0], [1]),
             compact=lambda: ctx.kvd_pages_compact(c.tuple, c.tuple, scratch),
             free=lambda: ctx.kvd_pages_free(c.tuple, [0, 1]),
             sample=lambda: ctx.kvd_scaffold_sample(x, 5000, 20, 5000, None, None, None, None, u, t))
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls[what]()
graph.replay()
assert ctx.kvd_poll_status() == 0
if what == "sample":
    got = t.tolist()
    calls[what]()
    assert got == t.tolist() and min(got) >= 0
if what == "grow":
    assert c.lens.tolist() == [71, 4] and first.tolist() == [70, 3]
print("fine")
"""


@pytest.mark.parametrize("what,shape,dtype", [("append", "qwen", 0), ("attend", "gemma", 0), ("attend", "smollm2", 1), ("grow", "qwen", 0), ("fork", "qwen", 0),
                                              ("sample", "smollm2", 0), ("sample", "smollm2", 1)])
def test_the_first_call_is_captured(what, shape, dtype):
    program = PROGRAM.format(root=ROOT, tests=os.path.join(ROOT, "tests"), shape=shape, dtype=dtype, what=what)
    r = subprocess.run([sys.executable, "-c", program], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("fine"), r.stdout[-2000:] + r.stderr[-2000:]
