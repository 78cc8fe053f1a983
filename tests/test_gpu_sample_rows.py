"""Sampling at every number of rows around those at which a row gets fewer CTAs: the token is the row's own."""
import re

import pytest
import torch

from test_gpu_cache4 import gen, open_ctx
from test_gpu_sample import like_a_model
from test_launch_rules import TEXT


def test_the_device_is_asked_how_many_rows_it_works_on_at_once():
    """Clusters of CTAs that fill an SM each are placed in groups of SMs, so that SMs over CTAs are more than fit at once; rows beyond that would
    wait for a second turn (17 rows of 49152 logits took 41 us with eight CTAs each, 22 with four)."""
    text = TEXT["kvd_sample.cu"]
    rule = text[text.index("static int ctas_of_a_row("):]
    rule = rule[:rule.index("}")]
    assert len(re.findall(r"m <= rows_at_once<F16, \d>\(ctx\)", rule)) == 2 and "num_sms" not in rule
    asked = text[text.index("static int rows_at_once("):text.index("static int ctas_of_a_row(")]
    assert "cudaOccupancyMaxActiveClusters(" in asked
    entry = text[text.index("kvd_scaffold_sample("):]
    assert "num_sms" not in entry and entry.count("ctas_of_a_row<") == 2


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [0, 1])
def test_rows_around_those_numbers(dtype):
    ctx, _ = open_ctx("smollm2", dtype)
    x = like_a_model(gen(31), 80, 9001, dtype)
    u, p = torch.rand(80, generator=gen(32), device="cuda"), torch.full((80,), 0.95, device="cuda")

    def tokens(m):
        out, probs = torch.full((81,), -7, dtype=torch.int32, device="cuda"), torch.full((81,), -7.0, device="cuda")
        ctx.kvd_scaffold_sample(x, x.stride(0), m, x.shape[1], None, None, p, None, u, out, probs)
        assert bool((out[m:] == -7).all()) and bool((probs[m:] == -7).all())
        return out[:m], probs[:m]

    whole = tokens(80)
    for m in (*range(1, 4), *range(12, 20), *range(30, 40), *range(70, 76)):
        assert all(torch.equal(a, b[:m]) for a, b in zip(tokens(m), whole))
    assert ctx.kvd_poll_status() == 0
