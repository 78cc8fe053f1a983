"""A batch of continuations of one prompt on a decoder stack, with caches ranked by accumulated attention weight.

The prompt is processed once.  Its keys' weights are taken while it is (kvd_prefill_attention_weights), every global layer's
keys are cut to a budget by them (kvd_cache_evict), and what is left is the shared prefix of the whole batch: each step attends
the prompt's keys once for all sequences and every sequence's own keys beside them (kvd_shared_prefix_attention).  One of the
continuations then goes on alone in a bounded cache of its own, which its decode steps rank (kvd_decode_attention_weights) and
evict from in place.  An evicted token is not lost: its residual row is checkpointed, and kvd_recompute_kv rebuilds its key and
value bit by bit when they are wanted after all.  Sliding-window layers keep their window as it is.

    python tests/session_shared_prompt.py [--prompt 2000] [--budget 512] [--batch 16] [--steps 32] [--alone 200] [--small]
Prints one JSON line per phase (full size: the 34-layer Gemma-3-4B-shaped stack, random weights).
"""
import argparse
import json
import os
import sys
import time

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "tests"))

import numpy as np  # noqa: E402
import torch  # noqa: E402

import paper_2603_19664_b200 as kvd  # noqa: E402
from kvd_synth import GEMMA3_4B_STACK, S_GEMMA, SEED_TOKENS  # noqa: E402
from stack_harness import GpuStack, torch_stack_weights  # noqa: E402

SINKS = 4  # the first tokens are never evicted


class SharedPromptStack(GpuStack):
    """`batch` continuations of at most `steps` tokens behind one prompt whose keys are cut to `budget` per global layer."""

    def __init__(self, stack, weights, batch, budget, steps, max_tokens, recent=32, device_weights=False):
        super().__init__(stack, weights, "full", 0, max_tokens, device_weights, tiled_attention=True)
        self.batch, self.keep, self.steps, self.recent = batch, budget, steps, recent
        s, dev = stack, dict(device="cuda")
        self.prompt_weights = [torch.zeros(max_tokens, **dev) if s.layer_shape(l).sliding_window == 0 else None for l in range(s.n_layers)]
        self.k_own = [torch.empty((batch, steps, self.kdim), dtype=torch.bfloat16, **dev) for _ in range(s.n_layers)]
        self.v_own = [torch.empty_like(k) for k in self.k_own]
        self.prefix = [None] * s.n_layers    # (k, v, row stride, first position, length)
        self.positions = [None] * s.n_layers  # of the prompt keys a global layer kept, by slot
        self.evicted = [None] * s.n_layers   # positions of the others, ascending

    def _attend(self, l, n, q, positions, positions_dev, segs, out):
        super()._attend(l, n, q, positions, positions_dev, segs, out)
        w = self.prompt_weights[l]
        if w is not None:
            p = positions[-1] + 1
            scratch = torch.empty(kvd.kvd_prefill_weights_scratch_bytes(self.ctx.desc, n, p), dtype=torch.uint8, device="cuda")
            self.ctx.kvd_prefill_attention_weights(l, n, q, positions_dev, segs, 0.0, w, w, p, scratch)

    def process_prompt(self, tokens):
        """Logits of the prompt's last token; the prompt's keys become the shared prefix."""
        logits = self.prefill(tokens)
        P = self.prompt = self.t
        for l in range(self.s.n_layers):
            k, v, window = self.k_live[l], self.v_live[l], self.s.layer_shape(l).sliding_window
            if window:  # what the window of a later token can still reach
                lo = max(0, P - window + 1)
                self.prefix[l] = (k[lo:], v[lo:], self.kdim, lo, P - lo)
                continue
            keep = min(self.keep, P)
            new = lambda dtype, *shape: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
            ko, vo, pos, w = new(k.dtype, keep, self.kdim), new(k.dtype, keep, self.kdim), new(torch.int32, keep), new(torch.float32, keep)
            slots, gone = new(torch.int32, keep), new(torch.int32, max(P - keep, 1))
            self.ctx.kvd_cache_evict(1, (k, v, None, self.prompt_weights[l], self.kdim, self.max_tokens), [P], keep, SINKS, [P - self.recent],
                                     (ko, vo, pos, w, self.kdim, keep), slots, gone, P - keep)
            # (a global layer sees every slot of it; positions of the tokens themselves are in the keys' rotation)
            self.prefix[l], self.positions[l], self.evicted[l] = (ko, vo, self.kdim, 0, keep), pos, gone[:P - keep]
            self.prompt_weights[l] = w
        return logits

    def step_batch(self, tokens, i):
        """Step i of the batch: tokens (DEVICE int32 [batch]) at position prompt + i; returns bf16 logits [batch, padded vocab]."""
        s, ctx, B, kd = self.s, self.ctx, self.batch, self.kdim
        pos = self.prompt + i
        pos_t = torch.full((B,), pos, dtype=torch.int32, device="cuda")
        h = torch.empty((B, s.d_hidden), dtype=torch.bfloat16, device="cuda")
        ctx.kvd_scaffold_embed(self.embed, tokens, B, s.d_hidden, s.vocab, h)
        for l in range(s.n_layers):
            q = self._queries(l, h, pos_t)
            k, v = self.k_own[l], self.v_own[l]
            ctx.kvd_recompute_kv(l, h, pos_t, B, k[0, i], v[0, i], self.steps * kd)
            out = torch.empty((B, s.n_q_heads, s.d_head), dtype=torch.bfloat16, device="cuda")
            ctx.kvd_shared_prefix_attention(l, B, q, [pos] * B, self.prefix[l], [[(k[b], v[b], kd, self.prompt, i + 1)] for b in range(B)], 0.0, out)
            h = self._after_attention(l, h, out)
        return self._linear(self.lin_head, h)

    def decode_batch(self, first_tokens, forced=None):
        """`steps` greedy steps (or over forced [steps][batch] tokens); tokens [steps][batch] and the last logits."""
        tok = torch.tensor(first_tokens, dtype=torch.int32, device="cuda")
        outs = []
        for i in range(self.steps):
            logits = self.step_batch(tok, i)
            nxt = torch.empty((self.batch,), dtype=torch.int32, device="cuda")
            self.ctx.kvd_scaffold_argmax(logits, logits.shape[1], self.batch, self.s.vocab, nxt)
            outs.append(nxt.tolist())
            tok = nxt if forced is None or i + 1 == self.steps else torch.tensor(forced[i], dtype=torch.int32, device="cuda")
        assert self.ctx.kvd_poll_status() == kvd.KVD_OK
        return outs, logits

    def go_on_alone(self, b, token, n_steps, room):
        """Sequence b goes on by itself for n_steps tokens; each global layer's cache holds at most keep + room keys and is cut
        back to `keep` in place whenever it is full.  Returns the tokens and, per global layer, the evicted positions."""
        s, ctx, kd, cap = self.s, self.ctx, self.kdim, self.keep + self.steps + room
        caches = []
        for l in range(s.n_layers):
            pk, pv, _, first, n = self.prefix[l]
            window = s.layer_shape(l).sliding_window
            size = n + self.steps + n_steps if window else max(cap, n + self.steps + 1)
            k, v = (torch.empty((size, kd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            k[:n], v[:n] = pk[:n], pv[:n]
            k[n:n + self.steps], v[n:n + self.steps] = self.k_own[l][b], self.v_own[l][b]
            c = dict(k=k, v=v, len=n + self.steps, first=first, window=window, gone=[])
            if not window:
                c["pos"], c["w"] = torch.empty(size, dtype=torch.int32, device="cuda"), torch.zeros(size, device="cuda")
                c["pos"][:n], c["w"][:n] = self.positions[l], self.prompt_weights[l]
                c["pos"][n:n + self.steps] = torch.arange(self.prompt, self.prompt + self.steps, dtype=torch.int32, device="cuda")
                c["slots"], c["out"] = torch.empty(size, dtype=torch.int32, device="cuda"), torch.empty(size, dtype=torch.int32, device="cuda")
                c["scratch"] = torch.empty(kvd.kvd_weights_scratch_bytes(ctx.desc, 1, size), dtype=torch.uint8, device="cuda")
            caches.append(c)
        tok, tokens = torch.tensor([token], dtype=torch.int32, device="cuda"), []
        for i in range(n_steps):
            pos = self.prompt + self.steps + i
            pos_t = torch.tensor([pos], dtype=torch.int32, device="cuda")
            h = torch.empty((1, s.d_hidden), dtype=torch.bfloat16, device="cuda")
            ctx.kvd_scaffold_embed(self.embed, tok, 1, s.d_hidden, s.vocab, h)
            for l, c in enumerate(caches):
                n = c["len"]
                q = self._queries(l, h, pos_t)
                # STORE_RESIDUAL of the row, and the new key and value behind the cached ones
                ctx.kvd_decode_step_kv(l, [], kd, h, pos_t, 1, [0], c["k"][n:], c["v"][n:], kd)
                out = torch.empty((1, s.n_q_heads, s.d_head), dtype=torch.bfloat16, device="cuda")
                c["len"] = n + 1
                if c["window"]:
                    ctx.kvd_decode_attention(l, 1, q, [pos], [[(c["k"], c["v"], kd, c["first"], n + 1)]], 0.0, out)
                else:
                    c["pos"][n], c["w"][n] = pos, 0.0
                    size = c["w"].numel()
                    # slots stand for positions: the layer sees all of them
                    ctx.kvd_decode_attention_weights(l, 1, q, [n], [[(c["k"], c["v"], kd, 0, n + 1)]], 0.0, out, c["w"], c["w"], size, n + 1, c["scratch"])
                    if n + 1 == size:
                        cache = (c["k"], c["v"], c["pos"], c["w"], kd, size)
                        ctx.kvd_cache_evict(1, cache, [n + 1], self.keep, SINKS, [pos + 1 - self.recent], cache, c["slots"], c["out"], size)
                        c["gone"].append(c["out"][:n + 1 - self.keep].clone())
                        c["len"] = self.keep
                h = self._after_attention(l, h, out)
            self._logits(h)
            tokens.append(self.greedy_token())
            tok = torch.tensor([tokens[-1]], dtype=torch.int32, device="cuda")
        assert ctx.kvd_poll_status() == kvd.KVD_OK
        return tokens, [torch.cat(c["gone"]) if c["gone"] else None for c in caches], caches


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--prompt", type=int, default=2000)
    ap.add_argument("--budget", type=int, default=512)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--alone", type=int, default=200)
    ap.add_argument("--small", action="store_true", help="small 6-layer stack instead of the 34-layer one")
    a = ap.parse_args()
    stack = S_GEMMA if a.small else GEMMA3_4B_STACK
    m = SharedPromptStack(stack, torch_stack_weights(stack), a.batch, a.budget, a.steps, a.prompt + a.steps + a.alone + 8, device_weights=True)
    rng = np.random.Generator(np.random.PCG64(SEED_TOKENS + 99))

    def timed(what, f, **more):
        torch.cuda.synchronize()
        t = time.perf_counter()
        got = f()
        torch.cuda.synchronize()
        print(json.dumps({"phase": what, "seconds": round(time.perf_counter() - t, 4), **more}), flush=True)
        return got

    timed("prompt", lambda: m.process_prompt(rng.integers(0, stack.vocab, size=a.prompt).tolist()), tokens=a.prompt, kept_per_global_layer=min(a.budget, a.prompt))
    outs, _ = timed("batch", lambda: m.decode_batch(rng.integers(0, stack.vocab, size=a.batch).tolist()), sequences=a.batch, steps=a.steps)
    _, gone, _ = timed("alone", lambda: m.go_on_alone(0, outs[-1][0], a.alone, 64), steps=a.alone)
    print(json.dumps({"evicted_per_global_layer": [int(g.numel()) for g in gone if g is not None][:1]}))


if __name__ == "__main__":
    main()
