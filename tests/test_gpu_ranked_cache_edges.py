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


# ------------------------------------------------------------------------------------------------ keys and values in one buffer
@pytest.mark.parametrize("dtype", [0, 2])
@pytest.mark.parametrize("cap,keep", [(300, 100), (5000, 1234)])
def test_evict_keys_and_values_of_one_buffer(dtype, cap, keep):
    """Rows that hold a token's key and its value, as the attention and rebuild calls take them: in place, into another such
    buffer, into one with the halves the other way round and into its second half of the slots."""
    nq, nkv, dh = SHAPES["smollm2"]
    ctx = kvd.Kvd(kvd.make_desc(1, 64, nq, nkv, dh, 1e-6, False, 1e-6))
    if dtype:
        ctx.kvd_set_dtype(dtype)
    dt = {0: torch.bfloat16, 2: torch.float32}[dtype]
    g, row, b = gen(cap), nkv * dh, 2
    stride = 2 * row + 16
    kv0 = rnd(g, b, 2 * cap, stride, dtype=dt)
    w = torch.rand((b, 2 * cap), generator=g, device="cuda")
    lens = [cap, cap - 3]
    want = [evict_plain(w[i].tolist(), list(range(2 * cap)), lens[i], keep, 4, 2**31) for i in range(b)]
    at = torch.tensor([x[0] for x in want], device="cuda")

    def rows_of(kv, first):
        return kv.gather(1, at[..., None].expand(b, keep, stride))[..., first:first + row]

    for form in ("in place", "another", "swapped", "behind"):
        kv = kv0.clone()
        cache = (kv, kv[:, :, row:], None, w, stride, 2 * cap)
        if form == "in place":
            to, ko, vo = cache[:2] + (None, None) + cache[4:], kv[:, :keep, :row], kv[:, :keep, row:2 * row]
        elif form == "behind":  # (one sequence: its rows end where the others begin)
            cache, to = (kv, kv[:, :, row:], None, w, stride, cap), (kv[0, cap:], kv[0, cap:, row:], None, None, stride, cap)
            ko, vo = kv[:1, cap:cap + keep, :row], kv[:1, cap:cap + keep, row:2 * row]
        else:
            other = torch.full_like(kv, 5.0)
            a, c = (0, row) if form == "another" else (row, 0)
            to = (other[:, :, a:], other[:, :, c:], None, None, stride, 2 * cap)
            ko, vo = other[:, :keep, a:a + row], other[:, :keep, c:c + row]
        n = 1 if form == "behind" else b
        slots, gone = torch.empty((b, 2 * cap), dtype=torch.int32, device="cuda"), torch.empty((b, 2 * cap), dtype=torch.int32, device="cuda")
        ctx.kvd_cache_evict(n, cache, lens[:n], keep, 4, None, to, slots, gone, 2 * cap)
        assert ctx.kvd_poll_status() == kvd.KVD_OK
        assert torch.equal(ko, rows_of(kv0, 0)[:n]) and torch.equal(vo, rows_of(kv0, row)[:n])
        if form == "in place":
            assert torch.equal(kv[:, :, 2 * row:], kv0[:, :, 2 * row:]) and torch.equal(kv[:, keep:], kv0[:, keep:])
        elif form == "behind":
            assert torch.equal(kv[:, :cap], kv0[:, :cap]) and torch.equal(kv[1:], kv0[1:])
        else:
            assert bool((other[:, :, 2 * row:] == 5.0).all()) and bool((other[:, keep:] == 5.0).all()) and torch.equal(kv, kv0)


def test_evict_refuses_rows_that_do_overlap():
    nq, nkv, dh = SHAPES["smollm2"]
    ctx = kvd.Kvd(kvd.make_desc(1, 64, nq, nkv, dh, 1e-6, False, 1e-6))
    row = nkv * dh
    kv, w = torch.zeros((2, 128, 2 * row), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 128), device="cuda")
    lists = (torch.empty((2, 128), dtype=torch.int32, device="cuda"), torch.empty((2, 128), dtype=torch.int32, device="cuda"))
    other = torch.zeros_like(kv)
    launches = ctx.kvd_launch_count()

    def no(cache, to):
        refused(B.KVD_ERR_INVALID_ARG, ctx.kvd_cache_evict, 2, cache, [64, 64], 10, 0, None, to, *lists, 128)

    whole = (kv, kv[:, :, row:], None, w, 2 * row, 64)
    no(whole, (other, other[:, :, row - 8:], None, None, 2 * row, 64))           # the value's columns begin in the key's
    no(whole, (other, other[:, :, 2 * row - 8:], None, None, 2 * row, 64))       # ... or end in the next key's
    no(whole, (other, other, None, None, 2 * row, 64))
    no(whole, (kv[:, :, row:], other, None, None, 2 * row, 64))                  # the cache's values as keys
    no(whole, (other, kv[:, 1:], None, None, 2 * row, 64))                       # its keys, a row on
    no(whole, (kv, kv[:, :, row:], None, None, 2 * row, 60))                     # in place with other strides
    no(whole, (kv[:, 8:], kv[:, 8:, row:], None, None, 2 * row, 64))
    no((kv, other, None, w, 2 * row, 64), (kv[:, :, row - 8:], torch.zeros_like(kv), None, None, 2 * row, 64))
    no((kv, other, None, w, row, 64), (kv[:, 32:], torch.zeros_like(kv), None, None, 2 * row, 64))  # other strides over the same rows
    assert ctx.kvd_launch_count() == launches


# ------------------------------------------------------------------------------------------------ a window without an end
@pytest.mark.parametrize("shape,rows,ctx_len", [("gemma", 64, 3000), ("smollm2", 300, 0), ("qwen", 700, 1500)])
@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 40, 2**30])
def test_prompt_weights_of_a_window_that_hides_nothing(shape, rows, ctx_len, window):
    """Windows up to the largest that a layer can have: cut into the launches of a layer without one, hence its bits."""
    nq, nkv, dh = SHAPES[shape]
    g, t = gen(rows), rows + ctx_len
    k, q = rnd(g, t, nkv, dh), rnd(g, rows, nq, dh)
    pos = torch.arange(ctx_len, t, dtype=torch.int32, device="cuda")
    got = []
    for w in (0, window):
        ctx, desc = open_ctx(shape, 0, w)
        scratch = torch.empty(kvd.kvd_prefill_weights_scratch_bytes(desc, rows, t), dtype=torch.uint8, device="cuda")
        got.append(torch.empty(t, device="cuda"))
        ctx.kvd_prefill_attention_weights(0, rows, q, pos, [(k, None, nkv * dh, 0, t)], 0.0, None, got[-1], t, scratch)
        assert ctx.kvd_poll_status() == kvd.KVD_OK
    assert abs(float(got[0].double().sum()) - rows * nq) < 1e-4 * rows * nq
    assert torch.equal(got[0], got[1])


# ------------------------------------------------------------------------------------------------ a prefix with values that are no numbers
@pytest.mark.parametrize("shape,dtype,copies,own", [("smollm2", 0, 1, 0), ("smollm2", 1, 6, 3), ("gemma", 0, 1, 1), ("gemma", 1, 3, 200), ("qwen", 0, 1, 2),
                                                    ("qwen", 1, 5, 200), ("g8-256", 0, 1, 90)])
@pytest.mark.parametrize("window", [0, 333])
def test_shared_prefix_with_values_that_are_not_finite(shape, dtype, copies, own, window):
    """A value of the prefix that is not finite, or a key, concerns the sequences that see it and nobody else: not those before
    it, those whose window has moved on, nor those that see other keys of the same block."""
    nq, nkv, dh = SHAPES[shape]
    prefix, first = 1500, 20
    q_pos = [19, 25, 700, 1395, 1399, 1400, 1519, 1600, 1732, 1733, 1740, 1853, 1900] * copies
    b, end = len(q_pos), first + prefix
    ctx, _ = open_ctx(shape, dtype, window, max_batch=b)
    g, row, dt = gen(53), nkv * dh, DT[dtype]
    pk, pv = rnd(g, prefix, nkv, dh, dtype=dt, std=0.5), rnd(g, prefix, nkv, dh, dtype=dt)
    k, v, q = rnd(g, b, 512, nkv, dh, dtype=dt, std=0.5), rnd(g, b, 512, nkv, dh, dtype=dt), rnd(g, b, nq, dh, dtype=dt)
    # own keys end at the query's token (or lie ahead of the prefix's tokens that the query does not see)
    own_at = [(max(end, p + 1 - own), p + 1) for p in q_pos]
    segs = [[(k[i], v[i], row, lo, hi - lo)] if hi > lo and own else [] for i, (lo, hi) in enumerate(own_at)]
    out = torch.empty_like(q)
    bad = 1400 - first
    for what in ("values", "keys"):
        pk2, pv2 = pk.clone(), pv.clone()
        if what == "values":
            pv2[bad, 0, 3], pv2[bad, nkv - 1, dh - 1] = math.inf, math.nan
        else:
            pk2[bad, 0, :2], pk2[bad, nkv - 1, 1] = math.inf, math.nan
        ctx.kvd_shared_prefix_attention(0, b, q, q_pos, (pk2, pv2, row, first, prefix), segs, 0.0, out)
        assert ctx.kvd_poll_status() == kvd.KVD_OK
        for i, p in enumerate(q_pos):
            at = torch.arange(first, end, device="cuda")
            n = own_at[i][1] - own_at[i][0] if segs[i] else 0
            seen = at <= p
            mine = torch.arange(own_at[i][0], own_at[i][0] + n, device="cuda")
            if window:
                seen, ours = seen & (at > p - window), mine > p - window
            else:
                ours = torch.ones(n, dtype=torch.bool, device="cuda")
            if bool(seen[bad]):
                if what == "values":  # in its channel of its KV head's queries, and there alone
                    group = nq // nkv
                    assert not bool(torch.isfinite(out[i, :group, 3]).any()) and not bool(torch.isfinite(out[i, nq - group:, dh - 1]).any())
                    assert int((~torch.isfinite(out[i])).sum()) == 2 * group
                continue
            seen = torch.cat([seen, ours])
            if not bool(seen.any()):
                assert not bool(out[i].any())
                continue
            p64 = softmax64(q[i], torch.cat([pk, k[i, :n]]), 1 / math.sqrt(dh), seen)
            close(out[i], out64(p64, torch.cat([pv, v[i, :n]])), O_TOL)


# ------------------------------------------------------------------------------------------------ several own segments behind a prefix
@pytest.mark.parametrize("shape,dtype", [("smollm2", 0), ("gemma", 0), ("gemma", 1), ("qwen", 0), ("qwen", 1), ("g1", 0), ("g8", 0), ("g8-256", 0)])
@pytest.mark.parametrize("window", [0, 250])
@pytest.mark.parametrize("copies", [1, 8])
def test_shared_prefix_ahead_of_several_own_segments(shape, dtype, window, copies):
    """Rebuilt keys, a window and the current token behind the prefix, as a bounded cache has them: with holes, segments of one
    key, keys ahead of the prefix, empty segments, and sequences whose live keys are a handful."""
    nq, nkv, dh = SHAPES[shape]
    prefix, first = 700, 50
    end = first + prefix
    cuts = [[(end, end + 300), (end + 300, end + 420), (end + 420, end + 421)], [(end, end + 1)], [(end + 3, end + 4), (end + 9, end + 10)],
            [(0, 40), (end, end + 130), (end + 200, end + 201), (end + 201, end + 202)], [], [(10, 50), (end + 100, end + 100), (end + 120, end + 128)],
            [(end, end + 64), (end + 70, end + 90)]]
    q_pos = [end + 420, end, end + 9, end + 201, end + 5, end + 127, end + 95]
    cuts, q_pos = cuts * copies, q_pos * copies
    b, cap = len(cuts), end + 500
    ctx, _ = open_ctx(shape, dtype, window, max_batch=b)
    g, row, dt = gen(61), nkv * dh, DT[dtype]
    pk, pv = rnd(g, prefix, nkv, dh, dtype=dt), rnd(g, prefix, nkv, dh, dtype=dt)
    k, v, q = rnd(g, b, cap, nkv, dh, dtype=dt), rnd(g, b, cap, nkv, dh, dtype=dt), rnd(g, b, nq, dh, dtype=dt)
    pos = torch.arange(cap, device="cuda")
    seen = torch.zeros((b, cap), dtype=torch.bool, device="cuda")
    for i, c in enumerate(cuts):
        seen[i, first:end] = True
        for lo, hi in c:
            seen[i, lo:hi] = True
        seen[i] &= pos <= q_pos[i]
        if window:
            seen[i] &= pos > q_pos[i] - window
    # own rows that nobody sees are not numbers
    k[~seen], v[~seen] = math.nan, math.inf
    segs = [segments(k[i], v[i], c, row) for i, c in enumerate(cuts)]
    out, joint = torch.empty_like(q), torch.empty_like(q)
    ctx.kvd_shared_prefix_attention(0, b, q, q_pos, (pk, pv, row, first, prefix), segs, 0.0, out)
    assert ctx.kvd_poll_status() == kvd.KVD_OK
    for i in range(b):
        kk, vv = k[i].clone(), v[i].clone()
        kk[first:end], vv[first:end] = pk, pv
        kk = torch.where(seen[i][:, None, None], kk, torch.zeros((), dtype=dt, device="cuda"))
        vv = torch.where(seen[i][:, None, None], vv, torch.zeros((), dtype=dt, device="cuda"))
        close(out[i], out64(softmax64(q[i], kk, 1 / math.sqrt(dh), seen[i]), vv), O_TOL)
    # the prefix listed among the segments of a call of its own, where there is room for it
    few = [i for i, c in enumerate(cuts) if len(c) < B.KVD_MAX_SEGMENTS][:7]
    ctx.kvd_decode_attention(0, len(few), q[few].contiguous(), [q_pos[i] for i in few], [[(pk, pv, row, first, prefix)] + segs[i] for i in few], 0.0, joint)
    assert ctx.kvd_poll_status() == kvd.KVD_OK
    for n, i in enumerate(few):
        close(out[i], joint[n].double(), 2 * O_TOL)


def test_indices_of_the_prompt_weights_hold_in_the_checking_build():
    """Their kernels test what they index (statistics, sums, partial columns) at several cuts of the work."""
    import os
    import subprocess
    import sys
    if os.environ.get("KVD_LIBRARY") == "check":
        pytest.skip("already the checking build")
    here = os.path.dirname(os.path.abspath(__file__))
    run = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", os.path.join(here, "test_gpu_ranked_cache.py"), os.path.abspath(__file__),
                          "-k", "test_prompt_weights and not refusals"], env=dict(os.environ, KVD_LIBRARY="check"), cwd=os.path.dirname(here),
                         capture_output=True, text=True, timeout=600)
    assert run.returncode == 0 and " passed" in run.stdout, run.stdout[-2000:] + run.stderr[-1000:]


# ------------------------------------------------------------------------------------------------ the exponential on the fp32 pipes
@pytest.mark.parametrize("upper", [False, True])
def test_exponential_on_the_fp32_pipes(upper):
    """Against 2^e in 64 bits.  From -126 to 127 the polynomial's 1.6e-7 (exact arithmetic, f = e - n is exact), the last step's
    rounding, 2^-24 of a value in [1, 2) or 2^-25 of one above 0.7, and the half of 2^-25 that the step before it leaves: 2.5e-7.  Between
    -127 and -126 results may lose their bits (2^-126), at and below -127 they are 0."""
    ctx, _ = open_ctx("g1")
    g = torch.Generator().manual_seed(71)
    whole = torch.arange(-126, 127, dtype=torch.float64)
    near = [0.0, 0.25, 0.5, 0.75] + [s * 2.0 ** -k for k in (3, 8, 12, 16, 20, 23) for s in (1, -1)] + [0.5 + s * 2.0 ** -k for k in (8, 12, 16, 20) for s in (1, -1)]
    e = torch.cat([(whole[:, None] + torch.tensor(near, dtype=torch.float64)[None]).flatten(), torch.rand(200000, generator=g, dtype=torch.float64) * 253 - 126,
                   torch.rand(100000, generator=g, dtype=torch.float64) * 2 - 1, -torch.exp(torch.rand(50000, generator=g, dtype=torch.float64) * 24 - 20)]).float()
    e = e[(e >= -126) & (e <= (127 if upper else 126.5))]
    inf, nan = math.inf, math.nan
    low = torch.cat([-126 - torch.rand(2000, generator=g), torch.tensor([-126.5, -126.25, -126.75])])
    low = low[(low > -127) & (low < -126)]
    none = torch.tensor([-127.0, -127.5, -128.0, -150.0, -1000.0, -1e30, -3.4e38, -inf])
    odd = torch.tensor([nan, -nan, inf] + ([127.0, 127.5, 128.0, 129.5, 1000.0, 1e30, 3.4e38] if upper else []))
    x = torch.cat([e, low, none, odd])
    x = torch.cat([x, x[:1]]) if x.numel() % 2 else x
    for shift in (0, 1):  # either half of a pair
        v = torch.roll(x, shift).cuda()
        out = torch.full_like(v, -1.0)
        ctx.kvd_selftest_exp2(v, out, upper)
        got = torch.roll(out.cpu(), -shift).double()
        a, b, c = e.numel(), e.numel() + low.numel(), e.numel() + low.numel() + none.numel()
        want = torch.exp2(e.double())
        off = ((got[:a] - want) / want).abs()
        assert float(off.max()) <= 2.5e-7, (float(off.max()), float(e[off.argmax()]))
        assert bool((got[a:b] >= 0).all()) and bool(((got[a:b] - torch.exp2(low.double())).abs() <= 2.0 ** -126).all())
        assert not bool(got[b:c].any())
        rest = got[c:c + odd.numel()]
        assert not bool((rest <= 1e30).any())
        if upper:
            assert bool((rest[3:] >= 2.0 ** 127).all()) and float(rest[2]) >= 2.0 ** 127


def test_exponential_refusals():
    ctx, _ = open_ctx("g1")
    x = torch.zeros(8, device="cuda")
    out, launches = torch.full_like(x, 7.0), ctx.kvd_launch_count()
    refused(B.KVD_ERR_INVALID_ARG, ctx.kvd_selftest_exp2, x[:3], out, False)
    refused(B.KVD_ERR_INVALID_ARG, ctx.kvd_selftest_exp2, x, None, False)
    refused(B.KVD_ERR_ALIGNMENT, ctx.kvd_selftest_exp2, x[1:7], out, False)
    ctx.kvd_selftest_exp2(x[:0], out, False)
    assert ctx.kvd_launch_count() == launches and bool((out == 7.0).all())
