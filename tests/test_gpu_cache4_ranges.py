"""Decode attention over a 4-bit cache where magnitudes lie far apart: scores at which fp32 no longer tells neighbours apart, and values of which
some blocks or tokens are many powers of two larger than others.  The bound is that of every block of 32 channels by itself.

Tolerances.  A weight is rounded to fp16 (2^-11 of itself), its product with the scale of its token and block again (2^-11), the output once.  Weights are
2^12 times as large as those of the definition over the largest of them, or more, before the division by their sum (which is 2^12 at least).  One that is
below 2^-14 all the same, 2^-26 of the largest, is off by 2^-25 instead: by 2^-37, times its value |v|.  The product is taken with the scale over U,
U = 2^-10 while none of the head's scales is 2^-9 or more, 1 while all of the block's are below 2, else a power of two between half the block's
largest scale S and S.  Where it is below 2^-14 (weight over the largest, times scale over U, below 2^-26) it is off by 2^-25, which is 2^-37 U in the output, times a step of at most 6.
So a block's error is at most
    (2^-10 + 2^-14) sum_j p_j |v_j| + half a step of the output + 2^-37 (sum of |v_j| over such weights + 6 U times the number of such products)
with 2^-14 for the scores' fp32 sums (256 products of magnitude 8 at most, in blocks of 32, 2^-24 of the running sum each, times ln 2).  Where scores are 2^18 or more
(as powers of two) the 2^12 may be lost."""
import math

import pytest
import torch

import paper_2603_19664_b200 as kvd
from test_gpu_cache4 import SHAPES, Cache, attend, attend64, gen, held, ints, open_ctx, rows

pytestmark = pytest.mark.gpu
DT = {0: torch.bfloat16, 1: torch.float16}
SHAPES.setdefault("g8-64", (8, 1, 64))
LN2 = 0.693147182464599609375  # the fp32 number that log2(e), rounded to fp32, takes to 1: scores are whole in powers of two


def per_block(got, q, k, v, scale, lost=False):
    group, (heads, dh) = got.shape[0] // k.shape[1], got.shape
    out, mass = attend64(q, k, v, scale)
    bits = 0 if lost else 12
    p = torch.softmax(torch.einsum("hd,thd->ht", q.double(), k.repeat_interleave(group, 1)) * scale, -1)
    rel = (p / p.amax(-1, keepdim=True)).T[:, :, None]                                                  # [tokens, heads, 1]
    top = v.abs().unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(group, 1)                          # [tokens, heads, blocks]: 4 to 6 times the scale
    most = top.amax(0) / 4
    U = torch.maximum(torch.where(most.amax(-1, keepdim=True) < 2**-9, 2**-10, 1.0), most)
    low = ((rel < 2.0**(-14 - bits)) * top).sum(0) + 6 * U * ((rel * (top / 6) / U < 2.0**(-14 - bits)) & (top > 0)).sum(0)
    bound = (2**-10 + 2**-14) * mass + torch.finfo(got.dtype).eps / 2 * out.abs() + torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
    bound = bound + (2.0**(-25 - bits) * low).repeat_interleave(32, 1)
    off = (got.double() - out).abs()
    assert bool((off <= bound).all()), float((off / bound).nan_to_num(1e9).max())


def run(shape, dtype, k, v, q, scale, lost=False):
    ctx, desc = open_ctx(shape, dtype)
    nq, nkv, dh = SHAPES[shape]
    n = k.shape[0]
    c = Cache(desc, [n], seed=n)
    ctx.kvd_cache4_append(0, c.tuple, [0], [n], ints(0), k, v, nkv * dh)
    hk, hv = held(k), held(v)
    for batch in (1, 64):  # (a tile or two a warp; many, over which the reference and the scales move)
        out = attend(ctx, desc, c, [0] * batch, q.expand(batch, -1, -1).contiguous(), 0, scale)
        assert ctx.kvd_poll_status() == 0
        for b in {0, batch // 2, batch - 1}:
            per_block(out[b], q[0], hk, hv, scale or 1 / math.sqrt(dh), lost)


# ------------------------------------------------------------------------------------------------ scores
@pytest.mark.parametrize("order", ["mixed", "rising", "falling", "one"])
@pytest.mark.parametrize("power", [10, 17, 18, 21, 22, 23, 24, 25, 26, 27, 28])
@pytest.mark.parametrize("shape,dtype", [("g1", 0), ("g1", 1), ("gemma", 0), ("g8-64", 1)])
def test_scores_whose_neighbours_are_far_apart(shape, dtype, power, order):
    """All scores are +-1.5 * 2^power, in powers of two, plus 0, 1, 2 or 4 times the distance of fp32's neighbours there, or times a half where that
    is less: every sum on the way is exact, so the weights are those of the definition.  700 keys (whole tiles and an end) and 37."""
    nq, nkv, dh = SHAPES[shape]
    for sign in (1, -1):
        for n in (700, 37):
            g = gen(power + n)
            pick = torch.randint(0, 4, (n,), generator=g, device="cuda")
            if order == "one":
                pick = torch.zeros(n, dtype=torch.long, device="cuda")
                pick[n // 3] = 3
            elif order != "mixed":
                pick = torch.sort(pick, descending=order == "falling")[0]
            step = torch.tensor([0.0, 1.0, 2.0, 4.0], device="cuda")[pick]
            unit = max(2.0 ** (power - 23), 0.5)
            big = power // 2
            k = torch.zeros((n, nkv, dh), device="cuda")
            k[:, :, 0], k[:, :, 32], k[:, :, 33] = sign * 1.5 * 2.0**big, step[:, None], 6.0  # (the 6 sets the scale and meets a 0)
            q = torch.zeros((1, nq, dh), device="cuda")
            q[:, :, 0], q[:, :, 32] = 2.0 ** (power - big), unit
            k, q = k.to(DT[dtype]), q.to(DT[dtype])
            assert torch.equal(held(k), k.double())
            run(shape, dtype, k, rows(power, n, nkv, dh, dtype), q, LN2, power >= 18)


# ------------------------------------------------------------------------------------------------ values
@pytest.mark.parametrize("shape,dtype", [("g1", 0), ("g1", 1), ("gemma", 0), ("gemma", 1), ("g8-64", 0), ("g8-64", 1), ("qwen", 0)])
@pytest.mark.parametrize("large", [6e4, 3e4, 1000.0, 20.0])
@pytest.mark.parametrize("where", ["start", "end", "all"])
def test_a_block_of_large_values_beside_small_ones(shape, dtype, large, where):
    """One block of a head holds large values, in the first tokens, the last ones or all; the others of the head 1e-3, 1e-2, ... : each is
    as exact as without it."""
    nq, nkv, dh = SHAPES[shape]
    for n in (600, 21):
        v = rows(5, n, nkv, dh, dtype).float().clamp(-3, 3) / 3
        v *= torch.tensor([1e-3, 1e-2, 1e-4, 0.3], device="cuda")[torch.arange(dh, device="cuda") // 32 % 4]
        some = {"start": slice(0, 5), "end": slice(n - 5, n), "all": slice(0, n)}[where]
        block = 1 if dh == 64 else 3
        v[some, :, 32 * block:32 * block + 32] = (rows(6, n, nkv, 32, dtype).float().clamp(-3, 3) / 3 * large)[some]
        run(shape, dtype, rows(7, n, nkv, dh, dtype), v.to(DT[dtype]), rows(8, 1, nq, dh, dtype), 0.0)


@pytest.mark.parametrize("shape,dtype", [("g1", 0), ("gemma", 1), ("g8-64", 0), ("qwen", 1)])
@pytest.mark.parametrize("at", [0, 333, 599])
def test_a_token_of_large_values_that_weighs_nothing(shape, dtype, at):
    """A token whose values are 2^25 times as large as the others', in all blocks, and whose weight is 0: the others come out as exact as without it."""
    nq, nkv, dh = SHAPES[shape]
    n = 600
    q = rows(11, 1, nq, dh, dtype)
    k = rows(12, n, nkv, dh, dtype, 0.3).float()
    k[at] = -8 * q[0].view(nkv, nq // nkv, dh)[:, 0].float()
    q = q.view(nkv, nq // nkv, dh)[:, :1].expand(nkv, nq // nkv, dh).reshape(1, nq, dh).contiguous()
    v = rows(13, n, nkv, dh, dtype, 1e-3).float()
    v[at] = 3e4
    run(shape, dtype, k.to(DT[dtype]), v.to(DT[dtype]), q, 0.0)


@pytest.mark.parametrize("dtype", [0, 1])
def test_blocks_of_every_size(dtype):
    """The blocks of a head are 2^4 apart, from the smallest scales to the largest, and each one's values change by 2^6 along the sequence."""
    nq, nkv, dh = SHAPES["gemma"]
    n = 900
    size = torch.exp2(4.0 * (torch.arange(dh, device="cuda") // 32) - (16 if dtype else 20))
    ramp = torch.exp2(6 * torch.linspace(-0.5, 0.5, n, device="cuda"))[:, None, None]
    v = rows(21, n, nkv, dh, 0).float() * size
    for along in (ramp, ramp.flip(0)):
        run("gemma", dtype, rows(22, n, nkv, dh, dtype), (v * along).clamp(-6e4, 6e4).to(DT[dtype]), rows(23, 1, nq, dh, dtype), 0.0)
