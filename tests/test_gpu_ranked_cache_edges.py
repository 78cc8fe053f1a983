"""Edges of the ranked cache and the shared prefix: protected slots beyond the budget, keys and values in one buffer, windows without
an end, values that are not finite behind a mask, several own segments behind a prefix.

Tolerances: those of the operators' other tests.  Weights: 4e-5 of the value; outputs of 16 bits: 1e-2 of the row in the 2-norm;
what is moved, counted or computed twice in the same order: equal."""
import math

import pytest
import torch

import paper_2603_19664_b200 as kvd
from paper_2603_19664_b200 import binding as B
from test_gpu_ranked_cache import DT, O_TOL, SHAPES, close, evict_plain, gen, open_ctx, out64, refused, rnd, segments, softmax64

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ more protected slots than stay
@pytest.mark.parametrize("kind", ["plain", "ties", "odd"])
@pytest.mark.parametrize("protected", ["all", "one more than stay", "half of them"])
@pytest.mark.parametrize("cap", [300, 1000, 2000, 3000, 8192, 9000, 40000])  # one launch; two; a cluster's slots dealt out
def test_evict_among_protected_slots(cap, protected, kind):
    """The selection that starts again among the protected slots, in place and into another cache, while another stream keeps SMs
    busy (CTAs of a cluster do not run at one pace)."""
    nq, nkv, dh = SHAPES["smollm2"]
    ctx, _ = open_ctx("smollm2")
    g, row, b = gen(cap), nkv * dh, 2
    keep = {"half of them": cap // 5}.get(protected, cap // 3)
    w = torch.rand((b, cap), generator=g, device="cuda")
    if kind == "ties":
        w = torch.floor(w * 4) / 4
    elif kind == "odd":
        w = torch.randn((b, cap), generator=g, device="cuda")
        w[:, ::7], w[:, 1::11], w[:, 2::13], w[:, 3::5], w[:, 4::9] = math.nan, math.inf, -math.inf, 0.0, -0.0
    pos = torch.stack([torch.randperm(cap, generator=g, device="cuda") for _ in range(b)]).to(torch.int32)
    k, v = rnd(g, b, cap, row), rnd(g, b, cap, row)
    lens = [cap, cap - 1]
    start = [{"all": -2**31, "one more than stay": cap - keep - 1, "half of them": cap // 2}[protected]] * b
    want = [evict_plain(w[i].tolist(), pos[i].tolist(), lens[i], keep, 0, start[i]) for i in range(b)]
    assert all(sum(p >= start[i] for p in pos[i, :lens[i]].tolist()) >= keep for i in range(b))
    at = torch.tensor([x[0] for x in want], dtype=torch.long, device="cuda")
    wide = at[..., None].expand(b, keep, row)
    want_k, want_v, want_pos, want_w = k.gather(1, wide), v.gather(1, wide), pos.gather(1, at.to(torch.int64)), w.gather(1, at)
    side, a = torch.cuda.Stream(), torch.ones((2048, 2048), device="cuda")
    for in_place in [True] * 8 + [False]:
        cache = (k.clone(), v.clone(), pos.clone(), w.clone(), row, cap)
        to = cache if in_place else (torch.zeros_like(k), torch.zeros_like(v), torch.zeros_like(pos), torch.zeros_like(w), row, cap)
        slots, gone = torch.full((b, cap), -9, dtype=torch.int32, device="cuda"), torch.full((b, cap), -9, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(4):
                torch.mm(a, a)
        ctx.kvd_cache_evict(b, cache, lens, keep, 0, start, to, slots, gone, cap)
        assert ctx.kvd_poll_status() == kvd.KVD_OK
        for i in range(b):
            assert slots[i, :keep].tolist() == want[i][0] and gone[i, :lens[i] - keep].tolist() == want[i][1]
        assert torch.equal(to[0][:, :keep], want_k) and torch.equal(to[1][:, :keep], want_v) and torch.equal(to[2][:, :keep], want_pos)
        assert torch.equal(to[3][:, :keep].view(torch.int32), want_w.view(torch.int32))
    torch.cuda.synchronize()
