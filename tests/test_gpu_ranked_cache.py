"""Attention weights of cached keys, eviction by them, and attention behind a shared prefix, against plain forms in 64 bits.

Tolerances.  A weight 2^(s - z) has the relative error of its exponent, ln 2 times the error of s - z: s = (q.k) * scale is an
fp32 sum of d_head exact products (at most d_head * 2^-24 of the sum of their magnitudes, in practice its root) and one rounding
of a number below 64 (2^-19), z likewise; 4e-5 covers d_head 256 and scores up to 64.  Outputs are rounded to 16 bits
(2^-9 for bf16), as are the softmax weights of the tensor-core kernels, so 1e-2 of the row in the 2-norm holds for both
types.  What is moved or counted is compared exactly."""
import math

import numpy as np
import pytest
import torch

import paper_2603_19664_b200 as kvd
from paper_2603_19664_b200 import binding as B

pytestmark = pytest.mark.gpu

SHAPES = {"smollm2": (9, 3, 64), "gemma": (8, 4, 256), "qwen": (32, 8, 128), "g1": (4, 4, 128), "g8": (16, 2, 64), "g8-256": (8, 1, 256)}
DT = {0: torch.bfloat16, 1: torch.float16}
W_TOL, O_TOL = 4e-5, 1e-2


def open_ctx(shape, dtype=0, window=0, max_batch=8, max_tokens=8192):
    nq, nkv, dh = SHAPES[shape]
    desc = kvd.make_desc(1, 64, nq, nkv, dh, 1e-6, False, 1e-6, max_tokens_per_seq=max_tokens, max_batch=max_batch)
    ctx = kvd.Kvd(desc)
    if dtype:
        ctx.kvd_set_dtype(dtype)
    ctx.kvd_set_layer(0, torch.zeros((64, 2 * nkv * dh), dtype=DT[dtype], device="cuda"), torch.ones(64, dtype=DT[dtype], device="cuda"), None, 1e4, window)
    ctx.kvd_attach_workspace(torch.empty(kvd.kvd_workspace_bytes(desc), dtype=torch.uint8, device="cuda"))
    return ctx, desc


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rnd(g, *shape, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def softmax64(q, k, scale, seen):
    """[heads, keys] weights of one query row (q [heads, d], k [keys, kv heads, d], seen [keys]); all zero where nothing is seen."""
    group = q.shape[0] // k.shape[1]
    s = torch.einsum("hd,thd->ht", q.double(), k.double().repeat_interleave(group, 1)) * scale
    s = torch.where(seen[None], s, torch.full_like(s, -math.inf))
    if not bool(seen.any()):
        return torch.zeros_like(s)
    return torch.softmax(s, -1)


def out64(p, v):
    v = torch.where((p.sum(0) > 0)[:, None, None], v.double(), torch.zeros((), dtype=torch.float64, device="cuda"))
    return torch.einsum("ht,thd->hd", p, v.repeat_interleave(p.shape[0] // v.shape[1], 1))


def close(got, want, tol):
    assert bool(torch.isfinite(got).all())
    d, n = (got.double() - want).norm(), want.norm()
    assert float(d) <= tol * float(n) + 1e-30, (float(d), float(n))


def close_weights(got, want):
    assert bool(torch.isfinite(got).all())
    off = (got.double() - want).abs()
    assert float((off / (want.abs() + 1e-6)).max()) <= W_TOL, float((off / (want.abs() + 1e-6)).max())


def segments(k, v, cuts, row):
    """Segments [a, b) of one buffer, positions as in the buffer."""
    return [(k[a:], v[a:], row, a, b - a) for a, b in cuts]


# ------------------------------------------------------------------------------------------------ weights of a decode step
@pytest.mark.parametrize("shape,dtype", [("smollm2", 0), ("gemma", 0), ("gemma", 1), ("qwen", 0), ("qwen", 1), ("g1", 0), ("g8", 0), ("g8-256", 0)])
@pytest.mark.parametrize("window", [0, 100])
def test_decode_weights(shape, dtype, window):
    nq, nkv, dh = SHAPES[shape]
    ctx, desc = open_ctx(shape, dtype, window)
    g, row = gen(3), nkv * dh
    # lengths from one key to several chunks; holes between segments; keys past the query; a sequence without keys
    cuts = [[(0, 1)], [(0, 33)], [(5, 200), (250, 251)], [], [(0, 700), (700, 1301)], [(64, 128), (300, 900), (900, 901), (1000, 1024)]]
    q_pos = [0, 40, 250, 7, 1290, 1023]
    cap, b = 1400, len(cuts)
    k, v = rnd(g, b, cap, nkv, dh, dtype=DT[dtype]), rnd(g, b, cap, nkv, dh, dtype=DT[dtype])
    q = rnd(g, b, nq, dh, dtype=DT[dtype])
    held = torch.zeros((b, cap), dtype=torch.bool, device="cuda")
    for i, c in enumerate(cuts):
        for lo, hi in c:
            held[i, lo:hi] = True
    pos = torch.arange(cap, device="cuda")
    seen = held & (pos[None] <= torch.tensor(q_pos, device="cuda")[:, None])
    if window:
        seen &= pos[None] > torch.tensor(q_pos, device="cuda")[:, None] - window
    # what is not seen is not numbers
    k[~seen], v[~seen] = math.nan, math.inf
    segs = [segments(k[i], v[i], c, row) for i, c in enumerate(cuts)]
    past = torch.rand((b, cap), generator=g, device="cuda")
    out, plain = torch.empty_like(q), torch.empty_like(q)
    weights = torch.full((b, cap + 3), -7.0, device="cuda")
    scratch = torch.empty(kvd.kvd_weights_scratch_bytes(desc, b, cap), dtype=torch.uint8, device="cuda")
    scale = 1.5 / math.sqrt(dh)
    past_wide = torch.nn.functional.pad(past, (0, 3))
    ctx.kvd_decode_attention_weights(0, b, q, q_pos, segs, scale, out, past_wide, weights, cap + 3, cap, scratch)
    ctx.kvd_decode_attention(0, b, q, q_pos, segs, scale, plain)
    assert ctx.kvd_poll_status() == kvd.KVD_OK
    assert torch.equal(out, plain)  # the bits of the call without weights
    for i in range(b):
        p = softmax64(q[i], torch.where(seen[i][:, None, None], k[i], torch.zeros((), dtype=k.dtype, device="cuda")), scale, seen[i])
        close_weights(weights[i, :cap], past[i].double() + p.sum(0))
        close(out[i], out64(p, v[i]), O_TOL)
    assert bool((weights[:, cap:] == -7.0).all())  # positions past n_positions are not written
    # without earlier weights, and in place
    again = torch.empty((b, cap), device="cuda")
    ctx.kvd_decode_attention_weights(0, b, q, q_pos, segs, scale, out, None, again, cap, cap, scratch)
    own = past.clone()
    ctx.kvd_decode_attention_weights(0, b, q, q_pos, segs, scale, out, own, own, cap, cap, scratch)
    assert torch.equal(own, weights[:, :cap]) and torch.equal(past + again, own)


def test_decode_weights_of_a_long_cache_and_a_large_batch():
    """More chunks than a warp's lanes take at once; more sequences than one launch describes; another stream."""
    ctx, desc = open_ctx("smollm2", max_batch=70, max_tokens=40000)
    nq, nkv, dh = SHAPES["smollm2"]
    g, b = gen(4), 70
    lens = [39000 if i == 69 else 1 + 13 * i for i in range(b)]
    k, v, q = rnd(g, 39000, nkv, dh), rnd(g, 39000, nkv, dh), rnd(g, b, nq, dh)
    segs = [[(k, v, nkv * dh, 0, n)] for n in lens]
    out, weights = torch.empty_like(q), torch.empty((b, 39000), device="cuda")
    scratch = torch.empty(kvd.kvd_weights_scratch_bytes(desc, b, 39000), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx.kvd_decode_attention_weights(0, b, q, [n - 1 for n in lens], segs, 0.0, out, None, weights, 39000, 39000, scratch)
        assert ctx.kvd_poll_status() == kvd.KVD_OK
    for i in (0, 1, 20, 63, 64, 69):
        p = softmax64(q[i], k[:lens[i]], 1 / 8, torch.ones(lens[i], dtype=torch.bool, device="cuda"))
        close_weights(weights[i, :lens[i]], p.sum(0))
        assert not bool(weights[i, lens[i]:].any())
        assert abs(float(weights[i].double().sum()) - nq) < 1e-4 * nq


def test_weights_of_scores_that_are_not_numbers():
    ctx, desc = open_ctx("qwen")
    nq, nkv, dh = SHAPES["qwen"]
    g = gen(5)
    k, v, q = rnd(g, 3, 100, nkv, dh), rnd(g, 3, 100, nkv, dh), rnd(g, 3, nq, dh).abs() + 0.1
    k[0, 10, 0] = math.nan            # heads 0-3 of sequence 0
    k[1, 20, 1] = -math.inf           # one key of heads 4-7 weighs nothing
    k[2, :, 2] = -math.inf            # heads 8-11 weigh nothing at all
    row, lens = nkv * dh, [100] * 3
    out, w = torch.empty_like(q), torch.empty((3, 100), device="cuda")
    scratch = torch.empty(kvd.kvd_weights_scratch_bytes(desc, 3, 100), dtype=torch.uint8, device="cuda")
    ctx.kvd_decode_attention_weights(0, 3, q, [99] * 3, [[(k[i], v[i], row, 0, 100)] for i in range(3)], 0.0, out, None, w, 100, 100, scratch)
    assert bool(torch.isnan(w[0]).all()) and bool(torch.isfinite(w[1:]).all())
    assert abs(float(w[1].double().sum()) - nq) < 1e-3 and abs(float(w[2].double().sum()) - (nq - 4)) < 1e-3
    pos = torch.full((1,), 99, dtype=torch.int32, device="cuda")
    for i in range(3):
        got = torch.empty(100, device="cuda")
        s2 = torch.empty(kvd.kvd_prefill_weights_scratch_bytes(desc, 1, 100), dtype=torch.uint8, device="cuda")
        ctx.kvd_prefill_attention_weights(0, 1, q[i:i + 1], pos, [(k[i], None, row, 0, 100)], 0.0, None, got, 100, s2)
        assert ctx.kvd_poll_status() == kvd.KVD_OK
        if i == 0:
            assert bool(torch.isnan(got).all())
        else:
            close_weights(got, w[i].double())


# ------------------------------------------------------------------------------------------------ weights of a prompt
def prompt64(q, q_pos, k, scale, held, window):
    total = torch.zeros(k.shape[0], dtype=torch.float64, device="cuda")
    pos = torch.arange(k.shape[0], device="cuda")
    group = q.shape[1] // k.shape[1]
    for h in range(q.shape[1]):
        s = q[:, h].double() @ k[:, h // group].double().T * scale
        seen = held[None] & (pos[None] <= q_pos[:, None].long())
        if window:
            seen &= pos[None] > q_pos[:, None].long() - window
        s = torch.where(seen, s, torch.full_like(s, -math.inf))
        p = torch.softmax(s, -1)
        total += torch.where(seen.any(1, keepdim=True), p, torch.zeros_like(p)).sum(0)
    return total


@pytest.mark.parametrize("shape,dtype", [("smollm2", 0), ("smollm2", 1), ("gemma", 0), ("qwen", 1), ("g1", 0), ("g8", 0), ("g8-256", 1)])
@pytest.mark.parametrize("rows,ctx_len,window", [(1, 0, 0), (1, 500, 0), (5, 127, 0), (43, 85, 64), (64, 3000, 0), (300, 0, 0), (700, 333, 200)])
def test_prompt_weights(shape, dtype, rows, ctx_len, window):
    nq, nkv, dh = SHAPES[shape]
    ctx, desc = open_ctx(shape, dtype, window)
    g, t = gen(rows * 7 + ctx_len), rows + ctx_len
    k, q = rnd(g, t, nkv, dh, dtype=DT[dtype]), rnd(g, rows, nq, dh, dtype=DT[dtype])
    pos = torch.arange(ctx_len, t, dtype=torch.int32, device="cuda")
    past, got = torch.rand(t, generator=g, device="cuda"), torch.empty(t, device="cuda")
    scratch = torch.empty(kvd.kvd_prefill_weights_scratch_bytes(desc, rows, t), dtype=torch.uint8, device="cuda")
    scale = 1.2 / math.sqrt(dh)
    ctx.kvd_prefill_attention_weights(0, rows, q, pos, [(k, None, nkv * dh, 0, t)], scale, past, got, t, scratch)
    assert ctx.kvd_poll_status() == kvd.KVD_OK
    close_weights(got, past.double() + prompt64(q, pos, k, scale, torch.ones(t, dtype=torch.bool, device="cuda"), window))
    own = past.clone()
    ctx.kvd_prefill_attention_weights(0, rows, q, pos, [(k, None, nkv * dh, 0, t)], scale, own, own, t, scratch)
    assert torch.equal(own, got)


@pytest.mark.parametrize("shape", ["smollm2", "gemma", "qwen"])
@pytest.mark.parametrize("window", [0, 150])
def test_prompt_weights_with_holes_and_positions_in_any_order(shape, window):
    nq, nkv, dh = SHAPES[shape]
    ctx, desc = open_ctx(shape, 0, window)
    g, rows, cap = gen(9), 200, 1300
    k, q = rnd(g, cap, nkv, dh), rnd(g, rows, nq, dh)
    pos = torch.randint(-1, 1500, (rows,), generator=g, device="cuda").to(torch.int32)
    pos[3], pos[4] = -5, 2**31 - 1
    cuts = [(100, 101), (130, 640), (640, 777), (900, 1250)]
    held = torch.zeros(cap, dtype=torch.bool, device="cuda")
    for lo, hi in cuts:
        held[lo:hi] = True
    want = prompt64(q, pos, torch.where(held[:, None, None], k, torch.zeros((), dtype=k.dtype, device="cuda")), 1 / math.sqrt(dh), held, window)
    # rows of a wider buffer, and what nobody holds is not numbers
    wide = torch.full((cap, nkv * dh + 24), math.nan, dtype=k.dtype, device="cuda")
    wide[:, :nkv * dh] = torch.where(held[:, None, None], k, torch.full((), math.nan, dtype=k.dtype, device="cuda")).view(cap, -1)
    got = torch.full((cap + 50,), 3.0, device="cuda")
    scratch = torch.empty(kvd.kvd_prefill_weights_scratch_bytes(desc, rows, cap + 50), dtype=torch.uint8, device="cuda")
    segs = [(wide[a:], None, nkv * dh + 24, a, b - a) for a, b in cuts]
    ctx.kvd_prefill_attention_weights(0, rows, q, pos, segs, 0.0, None, got, cap + 50, scratch)
    assert ctx.kvd_poll_status() == kvd.KVD_OK
    close_weights(got[:cap], want)
    assert not bool(got[cap:].any())
    # nobody asks, or nobody answers
    for n, s in ((0, segs), (rows, [])):
        got.fill_(3.0)
        ctx.kvd_prefill_attention_weights(0, n, q, pos, s, 0.0, None, got, cap + 50, scratch)
        assert not bool(got.any())


def test_prompt_weights_with_scores_of_any_size():
    """Scores in the hundreds, and a row whose later keys exceed its first ones by far: nothing overflows."""
    ctx, desc = open_ctx("g1")
    nq, nkv, dh = SHAPES["g1"]
    g, rows = gen(11), 130
    k, q = rnd(g, 600, nkv, dh, std=1.0), rnd(g, rows, nq, dh, std=1.0)
    k[:300] *= 0.01
    k[500:] *= 16
    q[64:] *= 8
    pos = torch.arange(470, 600, dtype=torch.int32, device="cuda")
    got = torch.empty(600, device="cuda")
    scratch = torch.empty(kvd.kvd_prefill_weights_scratch_bytes(desc, rows, 600), dtype=torch.uint8, device="cuda")
    ctx.kvd_prefill_attention_weights(0, rows, q, pos, [(k, None, nkv * dh, 0, 600)], 1.0, None, got, 600, scratch)
    assert ctx.kvd_poll_status() == kvd.KVD_OK
    want = prompt64(q, pos, k, 1.0, torch.ones(600, dtype=torch.bool, device="cuda"), 0)
    # scores up to 2^13: their rounding alone is 2^-11, hence the weights' tolerance
    assert float(((got.double() - want).abs() / (want + 1e-3)).max()) < 5e-3
    assert abs(float(got.double().sum()) - rows * nq) < 1e-3 * rows * nq


# ------------------------------------------------------------------------------------------------ eviction
def evict_plain(weights, positions, n, keep, below, start):
    keep = min(keep, n)
    w = [float("-inf") if x != x else x for x in weights[:n]]
    order = sorted(range(n), key=lambda j: (not (positions[j] < below or positions[j] >= start), -w[j], j))
    stay = set(order[:keep])
    movers = iter(sorted(j for j in stay if j >= keep))
    slots = [j if j in stay else next(movers) for j in range(keep)]
    return slots, [positions[j] for j in range(n) if j not in stay]


def cache_of(g, b, cap, row, kind, dtype=torch.bfloat16):
    w = torch.rand((b, cap), generator=g, device="cuda")
    if kind == "ties":
        w = torch.floor(w * 4) / 4
    elif kind == "odd":
        w = torch.randn((b, cap), generator=g, device="cuda")
        w[:, ::7], w[:, 1::11], w[:, 2::13], w[:, 3::5], w[:, 4::9] = math.nan, math.inf, -math.inf, 0.0, -0.0
    pos = torch.stack([torch.randperm(3 * cap, generator=g, device="cuda")[:cap] for _ in range(b)]).to(torch.int32)
    return rnd(g, b, cap, row, dtype=dtype), rnd(g, b, cap, row, dtype=dtype), pos, w


@pytest.mark.parametrize("shape", ["smollm2", "gemma"])
@pytest.mark.parametrize("kind", ["plain", "ties", "odd"])
@pytest.mark.parametrize("cap,keep", [(1, 0), (1, 1), (33, 7), (700, 512), (1025, 1), (3000, 2999), (5000, 1234), (9000, 4000)])
def test_evict(shape, kind, cap, keep):
    nq, nkv, dh = SHAPES[shape]
    ctx, _ = open_ctx(shape)
    g, row, b = gen(cap + keep), nkv * dh, 3
    k, v, pos, w = cache_of(g, b, cap, row, kind)
    lens = [cap, max(0, cap - 5), min(keep, cap) // 2]
    start = [3 * cap - 20, 3 * cap, -2**31]  # recent ones; none; everything is protected
    room = keep + 3
    k_out, v_out = torch.zeros((b, room, row), dtype=k.dtype, device="cuda"), torch.zeros((b, room, row), dtype=k.dtype, device="cuda")
    pos_out, w_out = torch.full((b, room), -9, dtype=torch.int32, device="cuda"), torch.full((b, room), -9.0, device="cuda")
    slots, gone = torch.full((b, room), -9, dtype=torch.int32, device="cuda"), torch.full((b, cap), -9, dtype=torch.int32, device="cuda")
    ctx.kvd_cache_evict(b, (k, v, pos, w, row, cap), lens, keep, 4, start, (k_out, v_out, pos_out, w_out, row, room), slots, gone, cap)
    # the same in place
    k2, v2, pos2, w2 = k.clone(), v.clone(), pos.clone(), w.clone()
    slots2, gone2 = torch.full((b, cap), -9, dtype=torch.int32, device="cuda"), torch.full_like(gone, -9)
    cache = (k2, v2, pos2, w2, row, cap)
    ctx.kvd_cache_evict(b, cache, lens, keep, 4, start, cache, slots2, gone2, cap)
    assert ctx.kvd_poll_status() == kvd.KVD_OK
    for i in range(b):
        n = min(keep, lens[i])
        want, evicted = evict_plain(w[i].tolist(), pos[i].tolist(), lens[i], keep, 4, start[i])
        assert slots[i].tolist() == want + [-9] * (room - n) and gone[i].tolist() == evicted + [-9] * (cap - len(evicted))
        at = torch.tensor(want, dtype=torch.long, device="cuda")
        assert torch.equal(k_out[i, :n], k[i][at]) and torch.equal(v_out[i, :n], v[i][at]) and torch.equal(pos_out[i, :n], pos[i][at])
        assert torch.equal(w_out[i, :n].view(torch.int32), w[i][at].view(torch.int32))
        assert not bool(k_out[i, n:].any()) and bool((pos_out[i, n:] == -9).all()) and bool((w_out[i, n:] == -9).all())
        assert slots2[i].tolist()[:n] == want and gone2[i].tolist() == gone[i].tolist()
        assert torch.equal(k2[i, :n], k_out[i, :n]) and torch.equal(v2[i, :n], v_out[i, :n])
        assert torch.equal(pos2[i, :n], pos_out[i, :n]) and torch.equal(w2[i, :n].view(torch.int32), w_out[i, :n].view(torch.int32))
        assert torch.equal(k2[i, n:], k[i, n:]) and torch.equal(w2[i, n:].view(torch.int32), w[i, n:].view(torch.int32))


def test_evict_the_longest_cache_and_the_lists_alone():
    ctx, _ = open_ctx("smollm2", max_batch=80)
    cap = 131072
    g = gen(21)
    w = torch.floor(torch.rand((2, cap), generator=g, device="cuda") * 1000)
    slots, gone = torch.empty((2, 40000), dtype=torch.int32, device="cuda"), torch.empty((2, cap), dtype=torch.int32, device="cuda")
    # without positions slot j holds position j; without rows, positions and weights there are the lists alone
    ctx.kvd_cache_evict(2, (None, None, None, w, 0, cap), [cap, cap - 1], 40000, 10, None, (None, None, None, None, 0, 40000), slots, gone, cap)
    for i, n in enumerate((cap, cap - 1)):
        want, evicted = evict_plain(w[i].tolist(), list(range(n)), n, 40000, 10, 2**31)
        assert slots[i].tolist() == want and gone[i, :len(evicted)].tolist() == evicted
    # more sequences than one launch describes
    b, cap, row = 70, 40, 192
    k, v, pos, w = cache_of(g, b, cap, row, "ties")
    slots, gone = torch.empty((b, cap), dtype=torch.int32, device="cuda"), torch.empty((b, cap), dtype=torch.int32, device="cuda")
    k0 = k.clone()
    cache, lens = (k, v, pos.clone(), w.clone(), row, cap), [cap - i % 3 for i in range(b)]
    ctx.kvd_cache_evict(b, cache, lens, 17, 0, None, cache, slots, gone, cap)
    for i in range(b):
        want, evicted = evict_plain(w[i].tolist(), pos[i].tolist(), lens[i], 17, 0, 2**31)
        assert slots[i, :17].tolist() == want and gone[i, :len(evicted)].tolist() == evicted
        assert torch.equal(k[i, :17], k0[i][torch.tensor(want, device="cuda")])


def test_evict_rows_of_an_fp32_context():
    nq, nkv, dh = SHAPES["smollm2"]
    ctx = kvd.Kvd(kvd.make_desc(1, 64, nq, nkv, dh, 1e-6, False, 1e-6))
    ctx.kvd_set_dtype(2)
    g, row = gen(22), nkv * dh
    k, v, pos, w = cache_of(g, 2, 300, row + 4, "plain", torch.float32)
    k0, w0, p0 = k.clone(), w.clone(), pos.clone()
    slots, gone = torch.empty((2, 300), dtype=torch.int32, device="cuda"), torch.empty((2, 300), dtype=torch.int32, device="cuda")
    cache = (k, v, pos, w, row + 4, 300)
    ctx.kvd_cache_evict(2, cache, [300, 299], 100, 0, None, cache, slots, gone, 300)
    assert ctx.kvd_poll_status() == kvd.KVD_OK
    for i, n in enumerate((300, 299)):
        want, _ = evict_plain(w0[i].tolist(), p0[i].tolist(), n, 100, 0, 2**31)
        at = torch.tensor(want, device="cuda")
        assert slots[i, :100].tolist() == want and torch.equal(k[i, :100, :row], k0[i][at][:, :row])
        assert torch.equal(k[i, :, row:], k0[i, :, row:])  # what lies between the rows stays


# ------------------------------------------------------------------------------------------------ shared prefix
@pytest.mark.parametrize("shape,dtype", [("smollm2", 0), ("gemma", 0), ("gemma", 1), ("qwen", 0), ("qwen", 1), ("g1", 0), ("g8", 0), ("g8-256", 0)])
@pytest.mark.parametrize("batch,prefix,first,own", [(1, 1, 0, 1), (3, 127, 0, 9), (5, 1000, 3, 200), (40, 2500, 0, 30), (70, 300, 0, 5)])
def test_shared_prefix(shape, dtype, batch, prefix, first, own):
    nq, nkv, dh = SHAPES[shape]
    ctx, _ = open_ctx(shape, dtype, max_batch=70)
    g, row, dt = gen(batch + prefix), nkv * dh, DT[dtype]
    # the prefix as rows of a wider buffer that holds no numbers outside them
    stride = row + 16
    pk, pv = (torch.full((prefix + 2, stride), math.nan, dtype=dt, device="cuda") for _ in range(2))
    pk[1:-1, :row], pv[1:-1, :row] = rnd(g, prefix, row, dtype=dt), rnd(g, prefix, row, dtype=dt)
    k, v, q = rnd(g, batch, own, nkv, dh, dtype=dt), rnd(g, batch, own, nkv, dh, dtype=dt), rnd(g, batch, nq, dh, dtype=dt)
    lens = [(own - 3 * i) % (own + 1) for i in range(batch)]  # some have no key of their own
    start = first + prefix
    segs = [[(k[i], v[i], row, start, n)] for i, n in enumerate(lens)]
    q_pos = [start + n - 1 if n else start for n in lens]
    out = torch.empty_like(q)
    ctx.kvd_shared_prefix_attention(0, batch, q, q_pos, (pk[1:], pv[1:], stride, first, prefix), segs, 0.0, out)
    assert ctx.kvd_poll_status() == kvd.KVD_OK
    for i in range(batch):
        kk = torch.cat([pk[1:-1, :row].reshape(prefix, nkv, dh), k[i, :lens[i]]])
        vv = torch.cat([pv[1:-1, :row].reshape(prefix, nkv, dh), v[i, :lens[i]]])
        close(out[i], out64(softmax64(q[i], kk, 1 / math.sqrt(dh), torch.ones(len(kk), dtype=torch.bool, device="cuda")), vv), O_TOL)


@pytest.mark.parametrize("shape", ["smollm2", "gemma", "qwen"])
@pytest.mark.parametrize("window", [0, 333])
def test_shared_prefix_that_sequences_see_in_part(shape, window):
    """Queries inside the prefix, before it, and beyond it by more than the window; scores that grow along the prefix."""
    nq, nkv, dh = SHAPES[shape]
    ctx, _ = open_ctx(shape, 0, window, max_batch=8)
    g, row, prefix, first = gen(31), nkv * dh, 1500, 20
    pk, pv = rnd(g, prefix, nkv, dh), rnd(g, prefix, nkv, dh)
    pk *= torch.linspace(0.1, 6.0, prefix, device="cuda")[:, None, None].to(pk.dtype)
    q_pos = [20, 19, 700, 1519, 1600, 1700, 1853, 4000]
    own = [[], [(0, 20)], [(0, 10)], [], [(1520, 1600)], [(1690, 1701)], [(1520, 1854)], [(3900, 3990)]]
    ko, vo, q = rnd(g, 4096, nkv, dh), rnd(g, 4096, nkv, dh), rnd(g, 8, nq, dh)
    segs = [segments(ko, vo, c, row) for c in own]
    out = torch.empty_like(q)
    ctx.kvd_shared_prefix_attention(0, 8, q, q_pos, (pk, pv, row, first, prefix), segs, 0.0, out)
    assert ctx.kvd_poll_status() == kvd.KVD_OK
    pos = torch.arange(4096, device="cuda")
    kk, vv = ko.clone(), vo.clone()
    kk[first:first + prefix], vv[first:first + prefix] = pk, pv
    for i in range(8):
        seen = (pos >= first) & (pos < first + prefix)
        for lo, hi in own[i]:
            seen |= (pos >= lo) & (pos < hi)
        seen &= pos <= q_pos[i]
        if window:
            seen &= pos > q_pos[i] - window
        if not bool(seen.any()):
            assert not bool(out[i].any())
        else:
            close(out[i], out64(softmax64(q[i], kk, 1 / math.sqrt(dh), seen), vv), O_TOL)
    # without a prefix, the bits of decode attention
    plain = torch.empty_like(q)
    ctx.kvd_shared_prefix_attention(0, 8, q, q_pos, (pk, pv, row, first, 0), segs, 0.0, out)
    ctx.kvd_decode_attention(0, 8, q, q_pos, segs, 0.0, plain)
    assert torch.equal(out, plain)


def test_shared_prefix_equal_calls_give_equal_bits():
    nq, nkv, dh = SHAPES["qwen"]
    ctx, _ = open_ctx("qwen", max_batch=64)
    g = gen(41)
    pk, pv, k, v, q = rnd(g, 5000, nkv, dh), rnd(g, 5000, nkv, dh), rnd(g, 64, 50, nkv, dh), rnd(g, 64, 50, nkv, dh), rnd(g, 64, nq, dh)
    outs = [torch.empty_like(q) for _ in range(20)]
    for o in outs:
        ctx.kvd_shared_prefix_attention(0, 64, q, [5049] * 64, (pk, pv, nkv * dh, 0, 5000), [[(k[i], v[i], nkv * dh, 5000, 50)] for i in range(64)], 0.0, o)
    assert ctx.kvd_poll_status() == kvd.KVD_OK
    assert all(torch.equal(outs[0], o) for o in outs)


def test_shared_prefix_in_a_workspace_that_is_nearly_full():
    """Own keys up to the longest sequence: the prefix gets the partial slots that are left."""
    nq, nkv, dh = SHAPES["smollm2"]
    ctx, _ = open_ctx("smollm2", max_batch=2, max_tokens=4096)
    g = gen(43)
    pk, pv, k, v, q = rnd(g, 3000, nkv, dh), rnd(g, 3000, nkv, dh), rnd(g, 2, 4096, nkv, dh), rnd(g, 2, 4096, nkv, dh), rnd(g, 2, nq, dh)
    out = torch.empty_like(q)
    ctx.kvd_shared_prefix_attention(0, 2, q, [7095] * 2, (pk, pv, nkv * dh, 0, 3000), [[(k[i], v[i], nkv * dh, 3000, 4096)] for i in range(2)], 0.0, out)
    assert ctx.kvd_poll_status() == kvd.KVD_OK
    for i in range(2):
        kk, vv = torch.cat([pk, k[i]]), torch.cat([pv, v[i]])
        close(out[i], out64(softmax64(q[i], kk, 1 / 8, torch.ones(len(kk), dtype=torch.bool, device="cuda")), vv), O_TOL)


# ------------------------------------------------------------------------------------------------ refusals
def refused(status, call, *args):
    with pytest.raises(B.KvdError) as e:
        call(*args)
    assert e.value.status == status, e.value


def test_refusals():
    nq, nkv, dh = SHAPES["smollm2"]
    ctx, desc = open_ctx("smollm2", max_batch=4)
    row = nkv * dh
    k, v, q = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((2, 64, row), (2, 64, row), (2, nq, dh)))
    out, w = torch.full_like(q, 5.0), torch.full((2, 64), 5.0, device="cuda")
    scratch = torch.empty(kvd.kvd_weights_scratch_bytes(desc, 2, 64), dtype=torch.uint8, device="cuda")
    segs = [[(k[i], v[i], row, 0, 64)] for i in range(2)]
    launches = ctx.kvd_launch_count()
    dec = ctx.kvd_decode_attention_weights
    refused(B.KVD_ERR_CAPACITY, dec, 0, 2, q, [63, 63], segs, 0.0, out, None, w, 64, 60, scratch)          # a visible key has no room
    refused(B.KVD_ERR_INVALID_ARG, dec, 0, 2, q, [63, 63], segs, 0.0, out, None, w, 32, 64, scratch)       # rows shorter than their positions
    refused(B.KVD_ERR_CAPACITY, dec, 0, 2, q, [63, 63], segs, 0.0, out, None, w, 64, 64, scratch[:256])
    refused(B.KVD_ERR_ALIGNMENT, dec, 0, 2, q, [63, 63], segs, 0.0, out, None, w, 64, 64, scratch[16:])
    odd = torch.zeros(1024, dtype=torch.uint8, device="cuda")[2:]
    refused(B.KVD_ERR_ALIGNMENT, dec, 0, 2, q, [63, 63], segs, 0.0, out, odd, w, 64, 64, scratch)
    refused(B.KVD_ERR_INVALID_ARG, dec, 1, 2, q, [63, 63], segs, 0.0, out, None, w, 64, 64, scratch)       # no such layer
    refused(B.KVD_ERR_CAPACITY, dec, 0, 5, q, [63] * 5, segs + segs + segs[:1], 0.0, out, None, w, 64, 64, scratch)
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    pre = ctx.kvd_prefill_attention_weights
    s2 = torch.empty(kvd.kvd_prefill_weights_scratch_bytes(desc, 2, 64), dtype=torch.uint8, device="cuda")
    refused(B.KVD_ERR_CAPACITY, pre, 0, 2, q, pos, segs[0], 0.0, None, w[0], 63, s2)
    refused(B.KVD_ERR_CAPACITY, pre, 0, 2, q, pos, segs[0], 0.0, None, w[0], 64, s2[:256])
    refused(B.KVD_ERR_ALIGNMENT, pre, 0, 2, q, pos, segs[0], 0.0, None, w[0], 64, s2[8:])
    refused(B.KVD_ERR_INVALID_ARG, pre, 0, 2, q, pos, segs[0] + [(k[1], None, row, 63, 1)], 0.0, None, w[0], 64, s2)  # overlap
    refused(B.KVD_ERR_INVALID_ARG, pre, 0, 2, q, pos, [(k[1], None, row - 8, 0, 1)], 0.0, None, w[0], 64, s2)
    sh = ctx.kvd_shared_prefix_attention
    prefix = (k[0], v[0], row, 0, 64)
    refused(B.KVD_ERR_INVALID_ARG, sh, 0, 1, q, [70], prefix, [[(k[1], v[1], row, 63, 5)]], 0.0, out)     # overlaps the prefix
    refused(B.KVD_ERR_ALIGNMENT, sh, 0, 1, q, [70], (k[0], v[0], row + 4, 0, 8), [[]], 0.0, out)
    refused(B.KVD_ERR_INVALID_ARG, sh, 0, 1, q, [-1], prefix, [[]], 0.0, out)
    refused(B.KVD_ERR_CAPACITY, sh, 0, 5, q, [70] * 5, prefix, [[]] * 5, 0.0, out)
    ev = ctx.kvd_cache_evict
    p = torch.zeros((2, 64), dtype=torch.int32, device="cuda")
    lists = (torch.empty((2, 64), dtype=torch.int32, device="cuda"), torch.empty((2, 64), dtype=torch.int32, device="cuda"))
    cache, other = (k, v, p, w, row, 64), (torch.zeros_like(k), torch.zeros_like(v), p.clone(), w.clone(), row, 64)
    refused(B.KVD_ERR_INVALID_ARG, ev, 2, cache, [65, 1], 3, 0, None, other, *lists, 64)                   # more keys than slots
    refused(B.KVD_ERR_CAPACITY, ev, 2, cache, [64, 64], 10, 0, None, other, *lists, 20)                    # no room for the evicted
    refused(B.KVD_ERR_CAPACITY, ev, 2, cache, [64, 64], 60, 0, None, other[:5] + (50,), *lists, 64)        # ... for the kept
    refused(B.KVD_ERR_INVALID_ARG, ev, 2, cache, [64, 64], 10, 0, None, other, lists[0], None, 64)
    refused(B.KVD_ERR_INVALID_ARG, ev, 2, (k, None, p, w, row, 64), [64, 64], 10, 0, None, other, *lists, 64)
    refused(B.KVD_ERR_INVALID_ARG, ev, 2, cache, [64, 64], 10, 0, None, (k, v, p, w, row, 32), *lists, 64)  # in place with other strides
    refused(B.KVD_ERR_INVALID_ARG, ev, 2, cache, [64, 64], 10, 0, None, (k[:, 1:], other[1], other[2], other[3], row, 62), *lists, 64)
    refused(B.KVD_ERR_ALIGNMENT, ev, 2, (k, v, p, w, row + 4, 32), [30, 30], 10, 0, None, other, *lists, 64)
    big = torch.zeros((1, 131073), device="cuda")
    refused(B.KVD_ERR_CAPACITY, ev, 1, (None, None, None, big, 0, 131073), [131073], 10, 0, None, (None, None, None, None, 0, 64),
            lists[0], torch.empty((1, 131073), dtype=torch.int32, device="cuda"), 131073)
    assert ctx.kvd_launch_count() == launches and bool((out == 5.0).all()) and bool((w == 5.0).all())
    refused(B.KVD_ERR_ALIGNMENT, ev, 2, cache[:3] + (odd, row, 64), [64, 64], 10, 0, None, other, *lists, 64)
    assert ctx.kvd_launch_count() == launches
    f32 = kvd.Kvd(kvd.make_desc(1, 64, nq, nkv, dh, 1e-6, False, 1e-6))
    f32.kvd_set_dtype(2)
    f32.kvd_set_layer(0, torch.zeros((64, 2 * row), device="cuda"), torch.ones(64, device="cuda"), None, 1e4)
    f32.kvd_attach_workspace(torch.empty(kvd.kvd_workspace_bytes(f32.desc), dtype=torch.uint8, device="cuda"))
    refused(B.KVD_ERR_UNSUPPORTED, f32.kvd_shared_prefix_attention, 0, 1, q, [70], prefix, [[]], 0.0, out)
    refused(B.KVD_ERR_UNSUPPORTED, f32.kvd_decode_attention_weights, 0, 1, q, [63], segs[:1], 0.0, out, None, w, 64, 64, scratch)
    refused(B.KVD_ERR_UNSUPPORTED, f32.kvd_prefill_attention_weights, 0, 2, q, pos, segs[0], 0.0, None, w[0], 64, s2)
    fresh = kvd.Kvd(kvd.make_desc(1, 64, nq, nkv, dh, 1e-6, False, 1e-6))
    refused(B.KVD_ERR_STATE, fresh.kvd_shared_prefix_attention, 0, 1, q, [70], prefix, [[]], 0.0, out)
    assert kvd.kvd_weights_scratch_bytes(desc, 0, 5) == 0 and kvd.kvd_prefill_weights_scratch_bytes(desc, 1, 0) == 0


def test_indices_hold_in_the_checking_build():
    """The four calls with the library whose kernels test what they index."""
    import os
    import subprocess
    import sys
    if os.environ.get("KVD_LIBRARY") == "check":
        pytest.skip("already the checking build")
    here = os.path.abspath(__file__)
    picks = ["test_decode_weights[0-gemma-0]", "test_decode_weights[100-qwen-0]", "test_prompt_weights[43-85-64-smollm2-0]", "test_evict[9000-4000-odd-smollm2]",
             "test_evict[700-512-ties-gemma]", "test_shared_prefix[40-2500-0-30-qwen-0]", "test_shared_prefix[5-1000-3-200-gemma-0]"]
    run = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", *[f"{here}::{p}" for p in picks]], env=dict(os.environ, KVD_LIBRARY="check"),
                         cwd=os.path.dirname(os.path.dirname(here)), capture_output=True, text=True, timeout=600)
    assert run.returncode == 0 and f"{len(picks)} passed" in run.stdout, run.stdout[-2000:] + run.stderr[-1000:]
