"""Lists with fewer entries than the batch has sequences are refused, in C's half of the binding and by ctypes alike (no GPU)."""
import pytest
import torch

from paper_2603_19664_b200 import binding as B
from test_binding_calls import SEEN, Slow, fake  # noqa: F401  (a fixture)

T = torch.zeros((8, 64))
SEG = (T, T[1], 64, 5, 2)
CACHE = (T, T[1], T[2], T[3], 64, 64)
CALLS = [
    lambda c: c.kvd_cache_evict(2, CACHE, [5], 3, 4, None, CACHE, T, T, 64),           # (a sequence without a length is no empty cache)
    lambda c: c.kvd_cache_evict(2, CACHE, [], 3, 4, None, CACHE, T, T, 64),
    lambda c: c.kvd_cache_evict(2, CACHE, [5, 5], 3, 4, [9], CACHE, T, T, 64),         # (... nor one whose positions are all protected)
    lambda c: c.kvd_cache_evict(1, CACHE, (), 3, 4, None, CACHE, T, T, 64),
    lambda c: c.kvd_cache_evict(2, CACHE, [5, 5, 5], 3, 4, None, CACHE, T, T, 64),     # too many
    lambda c: c.kvd_cache_evict(2, CACHE, [5, 5], 3, 4, [1, 2, 3], CACHE, T, T, 64),
    lambda c: c.kvd_shared_prefix_attention(0, 2, T, [7], SEG, [[SEG], [SEG]], 0.0, T),
    lambda c: c.kvd_decode_attention_weights(0, 2, T, [7], [[SEG], [SEG]], 0.0, T, None, T, 64, 64, T),
    lambda c: c.kvd_decode_attention(0, 2, T, [7], [[SEG], [SEG]], 0.0, T),
    lambda c: c.kvd_decode_step_kv(0, [], 64, T, T, 2, [1], T, T, 64),                 # (what lies behind the list is no sequence)
]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("slow", [False, True])
def test_a_list_of_another_length_than_the_batch_is_refused(fake, monkeypatch, call, slow):  # noqa: F811
    if slow:
        monkeypatch.setattr(B, "_calls", Slow())
    with pytest.raises(IndexError):
        call(fake)
    assert not SEEN


def test_empty_lists_of_an_empty_batch_pass(fake):  # noqa: F811
    fake.kvd_cache_evict(0, CACHE, [], 3, 4, None, CACHE, T, T, 64)
    fake.kvd_cache_evict(0, CACHE, [], 3, 4, [], CACHE, T, T, 64)
    assert len(SEEN) == 2
