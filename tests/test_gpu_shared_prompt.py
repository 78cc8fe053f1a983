"""The ranked cache and the shared prefix on whole stacks (tests/session_shared_prompt.py)."""
import numpy as np
import pytest
import torch

from kvd_synth import S_GEMMA, S_QWEN, S_SMOL, make_stack_weights
from session_shared_prompt import SINKS, SharedPromptStack
from stack_harness import GpuStack

pytestmark = pytest.mark.gpu


def prompt_of(stack, n, seed=0):
    return np.random.Generator(np.random.PCG64(77 + seed)).integers(0, stack.vocab, size=n).tolist()


@pytest.mark.parametrize("stack", [S_GEMMA, S_QWEN, S_SMOL], ids=lambda s: s.name)
def test_a_budget_that_holds_the_prompt_changes_no_logits(stack):
    """Every sequence of the batch, over forced tokens, against the full cache of one sequence: bf16 stacks, so the last
    logits agree as two kernels' roundings allow (1e-2 per layer's attention, carried through the layers)."""
    w, P, B, steps = make_stack_weights(stack), 150, 5, 6
    m = SharedPromptStack(stack, w, B, P, steps, 256)
    m.process_prompt(prompt_of(stack, P))
    g = np.random.Generator(np.random.PCG64(5))
    tokens = g.integers(0, stack.vocab, size=(steps, B))
    _, logits = m.decode_batch(tokens[0].tolist(), forced=tokens[1:].tolist())
    for b in range(B):
        one = GpuStack(stack, w, "full", 0, 256)
        one.prefill(prompt_of(stack, P))
        for i in range(steps):
            want = one.step(int(tokens[i, b]))
        got = logits[b, :stack.vocab].float()
        assert float((got - want).norm()) <= 3e-2 * float(want.norm()), (b, float((got - want).norm() / want.norm()))


@pytest.mark.parametrize("stack", [S_GEMMA, S_SMOL], ids=lambda s: s.name)
def test_bounded_caches_and_what_they_let_go(stack):
    w, P, B, steps, keep = make_stack_weights(stack), 200, 3, 4, 64
    m = SharedPromptStack(stack, w, B, keep, steps, 400, recent=16)
    m.process_prompt(prompt_of(stack, P, 1))
    layers = [l for l in range(stack.n_layers) if stack.layer_shape(l).sliding_window == 0]
    for l in layers:
        kept, gone = m.positions[l].tolist(), m.evicted[l].tolist()
        assert sorted(kept + gone) == list(range(P)) and gone == sorted(gone) and len(kept) == keep
        assert set(range(SINKS)) <= set(kept) and set(range(P - 16, P)) <= set(kept)
        # the others by weight, and nothing evicted outweighs what stayed
        weights = m.prompt_weights[l]
        assert abs(float(weights.sum())) > 0 and bool((weights >= 0).all())
        # an evicted token's key and value come back bit by bit from its residual row
        p = gone[len(gone) // 2]
        k, v = torch.empty((1, m.kdim), dtype=torch.bfloat16, device="cuda"), torch.empty((1, m.kdim), dtype=torch.bfloat16, device="cuda")
        m.ctx.kvd_recompute_kv(l, None, None, 1, k, v, m.kdim, seq=0, first_row=p)
        assert torch.equal(k[0], m.k_live[l][p]) and torch.equal(v[0], m.v_live[l][p])
    outs, _ = m.decode_batch([1, 2, 3])
    tokens, gone, caches = m.go_on_alone(1, outs[-1][1], 60, 12)
    assert len(tokens) == 60 and all(0 <= t < stack.vocab for t in tokens)
    for l in layers:
        c = caches[l]
        assert keep <= c["len"] <= keep + steps + 12 and gone[l].numel() >= 2 * (steps + 12 - 4)
        held, away = c["pos"][:c["len"]].tolist(), gone[l].tolist() + m.evicted[l].tolist()
        assert sorted(held + away) == list(range(P + steps + 60))  # every token is either cached or known to be gone
        # every query of every head has been handed out once over the positions it saw
        assert bool(torch.isfinite(c["w"][:c["len"]]).all())
