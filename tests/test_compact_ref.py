"""The references of tests/compact_ref.py against their own definitions, and what the library refuses without a device."""
import ctypes

import numpy as np
import pytest

from paper_2609_13285_b200 import binding as gb
from paper_2609_13285_b200 import build as gbuild
from tests import compact_ref as ref


@pytest.fixture(scope="module")
def lib():
    gbuild.build()
    return gb.load()


def rows():
    rng = np.random.default_rng(11)
    yield rng.standard_normal((200, 64)).astype(np.float32)
    yield (rng.standard_normal((50, 128)) * 10.0 ** rng.uniform(-6, 4, (50, 1))).astype(np.float32)
    yield (1000 + 0.01 * rng.standard_normal((50, 64))).astype(np.float32)
    yield np.full((3, 64), -2.7, dtype=np.float32)
    yield np.zeros((2, 64), dtype=np.float32)
    yield (rng.integers(0, 31, (40, 64)) * 0.5 - 3).astype(np.float32)         # many on the borders
    yield (rng.standard_normal((20, 64)) * 1e9).astype(np.float32)             # clamped


def test_codes_cover_every_row_and_are_the_nearest():
    for x in rows():
        c, s, z = ref.quantise(x)
        v = ref.widen(c, s, z)
        clipped = np.clip(x.astype(np.float64), -65504, 65504)
        # s = 0 only where the row is one f16 value; else the error is half a step at most
        assert np.all(np.abs(v - clipped) <= s.astype(np.float64)[:, None] / 2)
        assert np.all(z.astype(np.float64) <= clipped.min(axis=1))
        assert np.all(z.astype(np.float64) + 15 * s.astype(np.float64) >= clipped.max(axis=1))
        less = np.nextafter(s, np.float16(-np.inf)).astype(np.float64)
        assert np.all((s == 0) | (z.astype(np.float64) + 15 * less < clipped.max(axis=1)))
        assert np.array_equal(ref.unpack(ref.pack(c)), c)


def test_bf16_of_f64_is_rounded_once():
    from paper_2609_13285_b200 import workloads as wl
    rng = np.random.default_rng(12)
    x = np.concatenate([rng.standard_normal(20000) * 10.0 ** rng.uniform(-8, 8, 20000), [0.0, 1.0, -1.0, 1.00390625, 1.01171875, -1.01171875]])
    a = wl.bf16_bits_to_f32(ref.to_bf16_bits(x)).astype(np.float64)
    for step in (-1, 1):                                  # no neighbour is nearer
        near = wl.bf16_bits_to_f32((ref.to_bf16_bits(x).astype(np.int32) + step).astype(np.uint16)).astype(np.float64)
        assert np.all((np.abs(a - x) <= np.abs(near - x)) | (x == 0))
    assert ref.to_bf16_bits([1.00390625, 1.01171875]).tolist() == [0x3F80, 0x3F82]           # ties go to the even pattern
    just = 1.00390625 + 2.0 ** -40                        # over a border by less than f32 can hold
    assert ref.to_bf16_bits([just, -just, 2 * 1.00390625 - just]).tolist() == [0x3F81, 0xBF81, 0x3F80]


def test_a_row_with_a_nan_reads_as_nan():
    x = np.ones((2, 64), dtype=np.float32)
    x[1, 5] = np.nan
    v = ref.widen(*ref.quantise(x))
    assert np.isfinite(v[0]).all() and np.isnan(v[1]).all()


def test_eviction_keeps_the_first_of_the_order():
    rng = np.random.default_rng(5)
    for n, keep in ((1, 1), (1, 0), (10, 4), (40, 39), (40, 40), (33, 50)):
        w = rng.integers(0, 6, n).astype(np.float32)
        pos = rng.permutation(n).astype(np.int32)
        moves, new_w, new_p = ref.evict(w, pos, keep, n, 2, 3)
        k = min(keep, n)
        assert sorted(p for p in new_p if p >= 0) == sorted(set(new_p[:k])) and np.all(new_p[k:] == -1) and np.all(new_w[k:] == 0)
        assert all(to < k <= t for to, t in moves)
        # whoever left does not outweigh whoever stayed, outside the protected ones
        left = [t for t in range(n) if pos[t] not in new_p[:k]]
        stayed = [t for t in range(n) if pos[t] in new_p[:k] and not (pos[t] < 2 or pos[t] >= n - 3)]
        assert not left or not stayed or max(w[left]) <= min(w[stayed])


def test_null_handles_and_structs_are_refused(lib):
    q4, pool = gb.GvaQ4Cache(), gb.GvaCache()
    bad = gb.GVA_ERR_INVALID_ARG
    n = None
    assert lib.gva_append_cache_at(n, ctypes.byref(pool), n, n, n, n, 1, n, n) == bad
    assert lib.gva_q4_append(n, ctypes.byref(q4), n, n, n, n, 1, n, n) == bad
    assert lib.gva_q4_append_chunk(n, ctypes.byref(q4), n, n, n, n, n, 1, 1, n, n) == bad
    assert lib.gva_q4_widen(n, ctypes.byref(q4), ctypes.byref(pool), n, n, 1, 1, n, n) == bad
    assert lib.gva_q4_decode(n, ctypes.byref(q4), n, n, n, n, n, 0, 1, 1, 0, n, n) == bad
    assert lib.gva_attention_weights(n, ctypes.byref(pool), n, n, n, n, 1.0, n, n, 1, 1, 1, 1, n, n) == bad
    assert lib.gva_q4_attention_weights(n, ctypes.byref(q4), n, n, n, n, 1.0, n, n, 1, 1, 1, 1, n, n) == bad
    assert lib.gva_evict(n, ctypes.byref(pool), n, n, n, n, n, 0, 0, n, n, n, 1, n, 0, 1, 1, n, n) == bad
    assert lib.gva_q4_evict(n, ctypes.byref(q4), n, n, n, n, n, 0, 0, n, n, n, 1, n, 0, 1, 1, n, n) == bad
    assert gb.gva_q4_decode_workspace_bytes(None, 1, 1) == 0
    assert gb.gva_evict_workspace_bytes(None, 1, 1) == 0
