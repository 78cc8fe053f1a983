"""What the operators around a ranked cache are measured on: attention that also returns what every key weighed (one token
per sequence, and a whole prompt), eviction by those weights, and attention of a batch that shares a long prefix.

A case is a dict: ``op``, ``heads`` (a layer shape of ``HEADS``), ``dtype`` of queries, keys, values and outputs, and sizes:

  weights   ``batch`` sequences of up to ``keys`` cached keys, one query token each, in ``parts`` segments
  prompt    ``rows`` query tokens behind ``ctx`` earlier ones, over all ``ctx + rows`` keys; ``window`` of the layer (0: none)
  evict     ``batch`` caches of up to ``slots`` keys, of which ``keep`` stay
  shared    ``batch`` sequences behind one prefix of ``prefix`` keys, up to ``keys`` own keys each

Sequences of a batch are ragged.  ``run`` computes the operators by elementary torch operations in 32 bits, or, where ``own``
is true, makes the framework's calls.
"""
import math

import torch

own = False

# query heads, KV heads, d_head of the layers that the repository's configurations and tests use
HEADS = {"smollm2-135m": (9, 3, 64), "gemma3-4b": (8, 4, 256), "qwen3-4b": (32, 8, 128), "grouped-8": (32, 4, 128)}
DTYPES = {"bf16": (0, torch.bfloat16), "f16": (1, torch.float16)}
SINKS, RECENT = 4, 64   # first and last positions that an eviction never takes
MAX_TOKENS, MAX_BATCH = 65536, 64


def listed():
    return [
        # one short sequence of the smallest layer: launches and latency are all there is
        dict(name="weights_smol_100", op="weights", heads="smollm2-135m", dtype="bf16", batch=1, keys=100, parts=1),
        # a small batch under a bounded cache, keys in three segments (rebuilt, window, current)
        dict(name="weights_gemma_b4_2048", op="weights", heads="gemma3-4b", dtype="bf16", batch=4, keys=2048, parts=3),
        # the largest decode batch of long sequences
        dict(name="weights_qwen_b16_8192", op="weights", heads="qwen3-4b", dtype="bf16", batch=16, keys=8192, parts=1),
        # a short prompt
        dict(name="prompt_smol_300", op="prompt", heads="smollm2-135m", dtype="f16", rows=300, ctx=0, window=0),
        # the last rows of a long prompt look over all of it (an observation window ahead of an eviction)
        dict(name="prompt_gemma_64_of_16384", op="prompt", heads="gemma3-4b", dtype="bf16", rows=64, ctx=16320, window=0),
        # one user turn on a sliding-window layer
        dict(name="prompt_gemma_local_837", op="prompt", heads="gemma3-4b", dtype="bf16", rows=837, ctx=1100, window=1024),
        # a whole prompt: the largest number of products
        dict(name="prompt_qwen_4096", op="prompt", heads="qwen3-4b", dtype="bf16", rows=4096, ctx=0, window=0),
        # a small cache over its budget
        dict(name="evict_smol_700", op="evict", heads="smollm2-135m", dtype="bf16", batch=1, slots=700, keep=512),
        # a batch of prompts compressed to a quarter
        dict(name="evict_qwen_b8_8192", op="evict", heads="qwen3-4b", dtype="bf16", batch=8, slots=8192, keep=2001),
        # four continuations of one short prompt
        dict(name="shared_smol_b4_500", op="shared", heads="smollm2-135m", dtype="bf16", batch=4, prefix=500, keys=30),
        # few sequences behind one long document
        dict(name="shared_gemma_b8_32768", op="shared", heads="gemma3-4b", dtype="f16", batch=8, prefix=32749, keys=65),
        # the largest batch behind one system prompt
        dict(name="shared_qwen_b64_8192", op="shared", heads="qwen3-4b", dtype="bf16", batch=64, prefix=8192, keys=300),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of lo..hi."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["weights", "prompt", "prompt", "evict", "shared", "shared"])
    heads, dtype = rng.choice(sorted(HEADS)), rng.choice(["bf16", "bf16", "f16"])
    if op == "weights":
        batch = _log(rng, 1, 64)
        keys = _log(rng, 1, min(32768, 131072 // batch))
        return dict(op=op, heads=heads, dtype=dtype, batch=batch, keys=keys, parts=rng.randint(1, 3) if keys >= 64 else 1)
    if op == "prompt":
        rows = _log(rng, 1, 4096)
        ctx = rng.choice([0, _log(rng, 16, max(16, min(32768, 4096 * 2048 // rows - rows // 2)))])
        return dict(op=op, heads=heads, dtype=dtype, rows=rows, ctx=ctx, window=rng.choice([0, 0, _log(rng, 16, 2048)]))
    if op == "evict":
        batch = _log(rng, 1, 64)
        slots = _log(rng, 256, min(32768, 65536 // batch))
        return dict(op=op, heads=heads, dtype=dtype, batch=batch, slots=slots, keep=_log(rng, 100, slots * 3 // 4))
    batch = _log(rng, 1, 64)
    return dict(op=op, heads=heads, dtype=dtype, batch=batch, prefix=_log(rng, 64, min(32768, 524288 // batch)), keys=_log(rng, 1, 300))


def _ragged(batch, top, least=1):
    """Lengths of a batch's sequences: a few tokens shorter each."""
    return [max(least, top - (37 * b) % (top // 8 + 1)) for b in range(batch)]


def _lens(case):
    if case["op"] == "evict":
        return _ragged(case["batch"], case["slots"], case["keep"])
    return _ragged(case["batch"], case["keys"])


# ----------------------------------------------------------------------------------------------- what a program has in hand
_contexts = {}


def _context(case):
    """The library context of a layer (one per model in a program, kept with its workspace)."""
    import paper_2603_19664_b200 as kvd
    nq, nkv, dh = HEADS[case["heads"]]
    at = (case["heads"], case["dtype"], case.get("window", 0))
    if at not in _contexts:
        desc = kvd.make_desc(1, 64, nq, nkv, dh, 1e-6, False, 1e-6, max_tokens_per_seq=MAX_TOKENS, max_batch=MAX_BATCH)
        ctx = kvd.Kvd(desc)
        code, dt = DTYPES[case["dtype"]]
        if code:
            ctx.kvd_set_dtype(code)
        w = torch.zeros((64, 2 * nkv * dh), dtype=dt, device="cuda")
        ctx.kvd_set_layer(0, w, torch.ones(64, dtype=dt, device="cuda"), None, 1e6, case.get("window", 0))
        ctx.kvd_attach_workspace(torch.empty(kvd.kvd_workspace_bytes(desc), dtype=torch.uint8, device="cuda"))
        _contexts[at] = (ctx, desc, kvd)
    return _contexts[at]


class _Draws:
    """Queries and keys as attention layers have them: scores of deviation 1, and one key in fifty that every query leans to."""

    def __init__(self, case, seed):
        self.nq, self.nkv, self.dh = HEADS[case["heads"]]
        self.dt = DTYPES[case["dtype"]][1]
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.lean = torch.randint(0, 2, (self.nkv, self.dh), generator=self.g, device="cuda").float().mul_(2).sub_(1)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda")

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda")

    def queries(self, n):
        q = self.normal(n, self.nkv, self.nq // self.nkv, self.dh)
        return (q + 0.25 * self.lean[None, :, None]).reshape(n, self.nq, self.dh).to(self.dt)

    def keys(self, *shape):
        k = self.normal(*shape, self.nkv, self.dh)
        heavy = (self.uniform(*shape) < 0.02).float()[..., None, None]
        return (k + heavy * self.lean).to(self.dt)

    def values(self, *shape):
        return self.normal(*shape, self.nkv, self.dh).to(self.dt)

    def past(self, *shape):
        """Weights accumulated by earlier tokens: most are small, a few large."""
        return torch.exp(2.0 * self.normal(*shape) - 3.0)


def prepare(case, seed):
    D = _Draws(case, seed)
    dh, scale = D.dh, 1.0 / math.sqrt(D.dh)
    st = dict(case=case, scale=scale, ctx=_context(case) if own else None)
    if case["op"] == "weights":
        B, lens = case["batch"], _lens(case)
        cap = max(lens)
        k, v = D.keys(B, cap), D.values(B, cap)
        cuts = [[n * i // case["parts"] for i in range(case["parts"] + 1)] for n in lens]
        row = D.nkv * dh
        segs = [[(k[b, lo:], v[b, lo:], row, lo, hi - lo) for lo, hi in zip(c, c[1:])] for b, c in enumerate(cuts)]
        st.update(q=D.queries(B), k=k, v=v, lens=lens, lens_dev=torch.tensor(lens, device="cuda"), segs=segs, q_pos=[n - 1 for n in lens],
                  past=D.past(B, cap), out=torch.empty((B, D.nq, dh), dtype=D.dt, device="cuda"),
                  weights=torch.empty((B, cap), device="cuda"))
        if own:
            ctx, desc, kvd = st["ctx"]
            st["scratch"] = torch.empty(kvd.kvd_weights_scratch_bytes(desc, B, cap), dtype=torch.uint8, device="cuda")
    elif case["op"] == "prompt":
        R, C = case["rows"], case["ctx"]
        T = R + C
        k = D.keys(T)
        st.update(q=D.queries(R), k=k, pos=torch.arange(C, T, dtype=torch.int32, device="cuda"), past=D.past(T), weights=torch.empty(T, device="cuda"),
                  segs=[(k, k, D.nkv * dh, 0, T)])
        if own:
            ctx, desc, kvd = st["ctx"]
            st["scratch"] = torch.empty(kvd.kvd_prefill_weights_scratch_bytes(desc, R, T), dtype=torch.uint8, device="cuda")
    elif case["op"] == "evict":
        B, lens, keep = case["batch"], _lens(case), case["keep"]
        cap = max(lens)
        # a cache that has been evicted from before: positions in no order, weights with ties (zeros, small multiples of 1/64)
        w = D.past(B, cap)
        w = torch.where(w < 0.2, torch.floor(w * 64) / 64, w)
        pos = torch.stack([torch.randperm(2 * cap, generator=D.g, device="cuda")[:cap] for _ in range(B)]).to(torch.int32)
        row = D.nkv * dh
        st.update(k=D.keys(B, cap).view(B, cap, row), v=D.values(B, cap).view(B, cap, row), past=w, pos=pos, lens=lens, lens_dev=torch.tensor(lens, device="cuda"),
                  recent=[2 * cap - RECENT] * B, k_out=torch.empty((B, keep, row), dtype=D.dt, device="cuda"),
                  v_out=torch.empty((B, keep, row), dtype=D.dt, device="cuda"), pos_out=torch.empty((B, keep), dtype=torch.int32, device="cuda"),
                  weights=torch.empty((B, keep), device="cuda"), slots=torch.empty((B, keep), dtype=torch.int32, device="cuda"),
                  evicted=torch.full((B, cap - keep), -1, dtype=torch.int32, device="cuda"))
        st["cache"] = (st["k"], st["v"], pos, w, row, cap)
        st["cache_out"] = (st["k_out"], st["v_out"], st["pos_out"], st["weights"], row, keep)
    else:
        B, lens, P = case["batch"], _lens(case), case["prefix"]
        cap, row = max(lens), D.nkv * dh
        pk, pv, k, v = D.keys(P), D.values(P), D.keys(B, cap), D.values(B, cap)
        st.update(q=D.queries(B), pk=pk, pv=pv, k=k, v=v, lens=lens, lens_dev=torch.tensor(lens, device="cuda"), q_pos=[P + n - 1 for n in lens],
                  prefix=(pk, pv, row, 0, P), segs=[[(k[b], v[b], row, P, n)] for b, n in enumerate(lens)],
                  out=torch.empty((B, D.nq, dh), dtype=D.dt, device="cuda"))
    return st


# ----------------------------------------------------------------------------------------------- plain forms
def _softmax(s):
    e = torch.exp(s - s.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _plain_weights(st):
    k, v, q = st["k"], st["v"], st["q"]
    B, cap, nkv, dh = k.shape
    s = torch.einsum("bhgd,bthd->bhgt", q.view(B, nkv, -1, dh).float(), k.float()) * st["scale"]
    seen = torch.arange(cap, device="cuda")[None] < st["lens_dev"][:, None]
    p = _softmax(s.masked_fill(~seen[:, None, None], -math.inf))
    o = torch.einsum("bhgt,bthd->bhgd", p, v.float())
    return {"out": o.reshape(q.shape).to(q.dtype), "weights": st["past"] + p.sum((1, 2))}


def _plain_prompt(st):
    k, q, pos, window = st["k"], st["q"], st["pos"], st["case"]["window"]
    T, nkv, dh = k.shape
    R = q.shape[0]
    s = torch.matmul(q.view(R, nkv, -1, dh).permute(1, 2, 0, 3).reshape(nkv, -1, dh).float(), k.permute(1, 2, 0).float()).mul_(st["scale"])
    behind = pos[:, None] - torch.arange(T, device="cuda")[None]
    hidden = behind < 0
    if window:
        hidden = hidden | (behind >= window)
    s = s.view(nkv, -1, R, T).masked_fill_(hidden, -math.inf)
    return {"weights": st["past"] + _softmax(s).sum((0, 1, 2))}


def _plain_evict(st):
    k, v, w, pos, keep = st["k"], st["v"], st["past"], st["pos"], st["case"]["keep"]
    B, cap, row = k.shape
    at = torch.arange(cap, device="cuda")
    held = at[None] < st["lens_dev"][:, None]
    rank = held.int() + (held & ((pos < SINKS) | (pos >= st["recent"][0]))).int()
    order = torch.sort(w, dim=1, descending=True, stable=True)[1]
    order = order.gather(1, torch.sort(rank.gather(1, order), dim=1, descending=True, stable=True)[1])
    kept = torch.zeros_like(held).scatter_(1, order[:, :keep], True)
    movers = keep + torch.sort((~kept[:, keep:]).int(), dim=1, stable=True)[1]
    hole = ~kept[:, :keep]
    nth = (hole.cumsum(1) - 1).clamp(min=0, max=max(0, cap - keep - 1))
    slots = torch.where(hole, movers.gather(1, nth), at[:keep]) if cap > keep else at[:keep].expand(B, keep)
    gone = held & ~kept
    first = torch.sort((~gone).int(), dim=1, stable=True)[1][:, : cap - keep]
    evicted = torch.where(at[: cap - keep][None] < gone.sum(1, keepdim=True), pos.gather(1, first), torch.full_like(first, -1, dtype=torch.int32))
    wide = slots[..., None].expand(B, keep, row)
    return {"k": k.gather(1, wide), "v": v.gather(1, wide), "positions": pos.gather(1, slots), "weights": w.gather(1, slots), "slots": slots.to(torch.int32),
            "evicted": evicted}


def _plain_shared(st):
    k, v, q = st["k"], st["v"], st["q"]
    B, cap, nkv, dh = k.shape
    P = st["pk"].shape[0]
    qh = q.view(B, nkv, -1, dh).float()
    seen = torch.arange(cap, device="cuda")[None] < st["lens_dev"][:, None]
    own_s = torch.einsum("bhgd,bthd->bhgt", qh, k.float()).masked_fill(~seen[:, None, None], -math.inf)
    p = _softmax(torch.cat([torch.einsum("bhgd,thd->bhgt", qh, st["pk"].float()), own_s], -1) * st["scale"])
    o = torch.einsum("bhgt,thd->bhgd", p[..., :P], st["pv"].float()) + torch.einsum("bhgt,bthd->bhgd", p[..., P:], v.float())
    return {"out": o.reshape(q.shape).to(q.dtype)}


def run(st):
    op = st["case"]["op"]
    if not own:
        return {"weights": _plain_weights, "prompt": _plain_prompt, "evict": _plain_evict, "shared": _plain_shared}[op](st)
    ctx, desc, kvd = st["ctx"]
    if op == "weights":
        B, cap = st["past"].shape
        ctx.kvd_decode_attention_weights(0, B, st["q"], st["q_pos"], st["segs"], st["scale"], st["out"], st["past"], st["weights"], cap, cap, st["scratch"])
        return {"out": st["out"], "weights": st["weights"]}
    if op == "prompt":
        ctx.kvd_prefill_attention_weights(0, st["q"].shape[0], st["q"], st["pos"], st["segs"], st["scale"], st["past"], st["weights"], st["past"].numel(),
                                          st["scratch"])
        return {"weights": st["weights"]}
    if op == "evict":
        ctx.kvd_cache_evict(len(st["lens"]), st["cache"], st["lens"], st["case"]["keep"], SINKS, st["recent"], st["cache_out"], st["slots"], st["evicted"],
                            st["evicted"].shape[1])
        return {"k": st["k_out"], "v": st["v_out"], "positions": st["pos_out"], "weights": st["weights"], "slots": st["slots"], "evicted": st["evicted"]}
    ctx.kvd_shared_prefix_attention(0, len(st["lens"]), st["q"], st["q_pos"], st["prefix"], st["segs"], st["scale"], st["out"])
    return {"out": st["out"]}


# ----------------------------------------------------------------------------------------------- 64 bits, from the definition
def _attend64(q, k, scale):
    """Softmax weights [heads, keys] of one token (q [heads, d]) over the keys of its KV heads (k [keys, kv heads, d])."""
    group = q.shape[0] // k.shape[1]
    kd = k.double()
    s = torch.stack([kd[:, h // group] @ q[h].double() for h in range(q.shape[0])]) * scale
    return torch.softmax(s, -1)


def _values64(p, v):
    group = p.shape[0] // v.shape[1]
    vd = v.double()
    return torch.stack([p[h] @ vd[:, h // group] for h in range(p.shape[0])])


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "weights":
        out, weights = [], st["past"].double()
        for b, n in enumerate(st["lens"]):
            p = _attend64(st["q"][b], st["k"][b, :n], st["scale"])
            out.append(_values64(p, st["v"][b, :n]))
            weights[b, :n] += p.sum(0)
        return {"out": torch.stack(out), "weights": weights}
    if case["op"] == "prompt":
        q, k, pos = st["q"], st["k"], st["pos"].long()
        nq, nkv = q.shape[1], k.shape[1]
        weights = st["past"].double()
        last = torch.arange(k.shape[0], device="cuda")
        for r0 in range(0, q.shape[0], 1024):
            p_r = pos[r0:r0 + 1024, None]
            seen = (last <= p_r) & (last > p_r - case["window"] if case["window"] else last >= 0)
            for h in range(nq):
                s = q[r0:r0 + 1024, h].double() @ k[:, h * nkv // nq].double().T * st["scale"]
                weights += torch.softmax(torch.where(seen, s, -math.inf), -1).sum(0)
        return {"weights": weights}
    if case["op"] == "evict":
        got = {name: [] for name in ("k", "v", "positions", "weights", "slots", "evicted")}
        keep = case["keep"]
        for b, n in enumerate(st["lens"]):
            w, pos = st["past"][b, :n].tolist(), st["pos"][b, :n].tolist()
            best = sorted(range(n), key=lambda j: (not (pos[j] < SINKS or pos[j] >= st["recent"][b]), -w[j], j))[:keep]
            stay = set(best)
            movers = iter(sorted(j for j in best if j >= keep))
            slots = [j if j in stay else next(movers) for j in range(keep)]
            gone = [pos[j] for j in range(n) if j not in stay]
            at = torch.tensor(slots, device="cuda")
            got["k"].append(st["k"][b][at].double())
            got["v"].append(st["v"][b][at].double())
            got["positions"].append([pos[j] for j in slots])
            got["weights"].append(torch.tensor([w[j] for j in slots], dtype=torch.float64))
            got["slots"].append(slots)
            got["evicted"].append(gone + [-1] * (max(st["lens"]) - keep - len(gone)))
        return {name: torch.stack(x) if torch.is_tensor(x[0]) else torch.tensor(x) for name, x in got.items()}
    out = []
    for b, n in enumerate(st["lens"]):
        k, v = torch.cat([st["pk"], st["k"][b, :n]]), torch.cat([st["pv"], st["v"][b, :n]])
        out.append(_values64(_attend64(st["q"][b], k, st["scale"]), v))
    return {"out": torch.stack(out)}


# ----------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    nq, nkv, dh = HEADS[case["heads"]]
    row = 2 * nkv * dh  # bytes of a key
    if case["op"] == "prompt":
        R, C, W = case["rows"], case["ctx"], case["window"]
        pairs = sum(min(C + r + 1, W) if W else C + r + 1 for r in range(R))
        first = max(0, C - W + 1) if W else 0
        # every visible score once
        return {"bytes": R * nq * dh * 2 + (C + R - first) * row + 8 * (C + R), "flops": 2 * dh * nq * pairs}
    lens, B = _lens(case), case["batch"]
    if case["op"] == "weights":
        n = sum(lens)
        return {"bytes": 2 * n * row + 4 * B * nq * dh + 8 * B * max(lens), "flops": 4 * dh * nq * n}
    if case["op"] == "evict":
        kept = B * case["keep"]
        return {"bytes": 4 * kept * row + 8 * sum(lens) + 12 * kept + 4 * (sum(lens) - kept), "flops": 0}
    n = sum(lens)
    return {"bytes": 2 * (n + case["prefix"]) * row + 4 * B * nq * dh, "flops": 4 * dh * nq * (n + B * case["prefix"])}
