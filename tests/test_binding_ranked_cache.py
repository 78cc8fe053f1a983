"""The calls of the ranked cache and the shared prefix: marshalled in C as by ctypes (no GPU: callbacks stand in for the library)."""
import ctypes

import pytest
import torch

import test_binding_calls as base
from paper_2603_19664_b200 import binding as B
from test_binding_calls import SEEN, Slow, fake  # noqa: F401  (a fixture)

T = torch.zeros((8, 64))
SEG = (T, T[1], 1 << 33, 5, 2)
ARRAYS = {
    "kvd_shared_prefix_attention": {4: (2, ctypes.c_int32), 5: (lambda a: 1, B.kvd_kv_segment), 6: (lambda a: a[2] * a[7], B.kvd_kv_segment)},
    "kvd_decode_attention_weights": {4: (2, ctypes.c_int32), 5: (lambda a: a[2] * a[6], B.kvd_kv_segment)},
    "kvd_prefill_attention_weights": {5: (6, B.kvd_kv_segment)},
    "kvd_cache_evict": {2: (lambda a: 1, B.kvd_ranked_cache), 3: (1, ctypes.c_int32), 6: (1, ctypes.c_int32), 7: (lambda a: 1, B.kvd_ranked_cache)},
}
CACHE, OTHER = (T, T[1], T[2], T[3], 64, 1 << 33), (None, None, T[5], None, 1 << 34, 9)
CALLS = [
    lambda c: c.kvd_shared_prefix_attention(1, 2, T, [7, 8], SEG, [[SEG], []], 0.25, T[2]),
    lambda c: c.kvd_shared_prefix_attention(1, 1, T, (7,), (123456, 4096, 64, 0, 3), [[SEG, SEG]], 0.25, T[2], stream=5),
    lambda c: c.kvd_decode_attention_weights(0, 2, T, [1, 2], [[SEG], [SEG, SEG]], 0.5, T[1], None, T[2], 1 << 40, 77, T[3]),
    lambda c: c.kvd_decode_attention_weights(0, 1, T, [1], [[]], 1, T[1], T[4], T[2], 64, 64, T[3]),
    lambda c: c.kvd_prefill_attention_weights(3, 9, T, T[1], [SEG, (T, None, 64, 0, 4)], 0.0, T[2], T[2], 100, T[3]),
    lambda c: c.kvd_prefill_attention_weights(3, 9, T, T[1], [SEG], 0.0, None, T[2], 100, T[3]),
    lambda c: c.kvd_cache_evict(2, CACHE, [5, 6], 3, 4, [10, -11], OTHER, T[6], T[7], 1 << 35),
    lambda c: c.kvd_cache_evict(1, CACHE, [5], 3, -4, None, CACHE, T[6], None, 0),
]


@pytest.fixture(autouse=True)
def arrays(monkeypatch):
    monkeypatch.setattr(base, "ARRAYS", {**base.ARRAYS, **ARRAYS})


@pytest.mark.parametrize("call", CALLS)
def test_the_library_is_handed_the_same(fake, monkeypatch, call):  # noqa: F811
    call(fake)
    with monkeypatch.context() as m:
        m.setattr(B, "_calls", Slow())
        call(fake)
    assert len(SEEN) == 2 and SEEN[0] == SEEN[1]


def test_values_arrive(fake):  # noqa: F811
    CALLS[6](fake)
    name, a = SEEN[0]
    assert name == "kvd_cache_evict" and a[1] == 2 and a[4:6] == [3, 4] and a[8:11] == [T[6].data_ptr(), T[7].data_ptr(), 1 << 35]
    c, o = B.kvd_ranked_cache.from_buffer_copy(a[2]), B.kvd_ranked_cache.from_buffer_copy(a[7])
    assert (c.k, c.v, c.positions, c.weights, c.row_stride, c.slots) == (*(T[i].data_ptr() for i in range(4)), 64, 1 << 33)
    assert (o.k, o.v, o.positions, o.weights, o.row_stride, o.slots) == (None, None, T[5].data_ptr(), None, 1 << 34, 9)
    assert list((ctypes.c_int32 * 2).from_buffer_copy(a[6])) == [10, -11]
    CALLS[2](fake)
    name, a = SEEN[1]
    assert a[9] is None and a[10] == T[2].data_ptr() and a[11:13] == [1 << 40, 77] and a[14] == T[3].numel() * 4


@pytest.mark.parametrize("call,error", [
    (lambda c: c.kvd_shared_prefix_attention(0, 1, T, [1], (T, T, 64, 0), [[]], 0.0, T), ValueError),
    (lambda c: c.kvd_cache_evict(1, CACHE[:5], [1], 1, 0, None, CACHE, T, T, 1), ValueError),
    (lambda c: c.kvd_cache_evict(1, CACHE, [1], "1", 0, None, CACHE, T, T, 1), ctypes.ArgumentError),
    (lambda c: c.kvd_decode_attention_weights(0, 2, T, [1], [[SEG]], 0.0, T, None, T, 64, 64, T), IndexError),
])
def test_what_is_no_argument_is_refused_either_way(fake, monkeypatch, call, error):  # noqa: F811
    for slow in (False, True):
        with monkeypatch.context() as m:
            if slow:
                m.setattr(B, "_calls", Slow())
            with pytest.raises(error):
                call(fake)
    assert not SEEN
