"""A whole decode step over a 4-bit cache whose pool is full."""
import pytest
import torch

import paper_2603_19664_b200 as kvd
from kvd_synth import S_GEMMA, S_QWEN, S_SMOL, make_stack_weights
from paper_2603_19664_b200 import binding as B
from session_sampled_answers import SampledAnswersStack
from test_gpu_cache4 import gen, ints
from test_gpu_sampled_answers import limits, prompt_of

pytestmark = pytest.mark.gpu
PAGE = kvd.KVD_PAGE_TOKENS


@pytest.mark.parametrize("stack", [S_GEMMA, S_QWEN, S_SMOL], ids=lambda s: s.name)
def test_a_whole_step_that_finds_no_page_says_so(stack):
    """The step goes on with positions of -1 in its norms and rotations; the status is still that of the pool, once."""
    w, P, answers = make_stack_weights(stack), 120, 3
    m = SampledAnswersStack(stack, w, answers, 2 + answers, 256)
    m.limits = limits(answers)
    m.process(0, prompt_of(stack, P))
    draws = torch.rand((PAGE, answers), generator=gen(1), device="cuda")
    m.u.copy_(draws[0])
    m.fork()
    m.decode(draws[1:9])
    assert m.cache[2].tolist() == [P] + [2 * PAGE] * answers and m.first.tolist() == [2 * PAGE - 1] * answers
    before = [x.clone() for x in m.cache[:4]]
    m.step_answers()
    assert m.first.tolist() == [-1] * answers
    assert m.ctx.kvd_poll_status() == B.KVD_ERR_CAPACITY and m.ctx.kvd_poll_status() == kvd.KVD_OK
    assert all(torch.equal(a, b) for a, b in zip(before, m.cache[:4]))
    # a position out of range by itself is still one
    m.ctx.kvd_recompute_kv(0, torch.zeros((1, stack.d_hidden), dtype=torch.bfloat16, device="cuda"), ints(-1), 1, m.k_new, m.v_new, m.kdim)
    assert m.ctx.kvd_poll_status() == B.KVD_ERR_POSITION
