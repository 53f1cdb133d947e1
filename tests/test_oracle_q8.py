"""The 64-bit statements of the 8-bit cache, of joining and of packed attention, pinned by closed forms."""
import numpy as np

from oracle import fp8
from oracle import kv as ref


def test_codes_and_scales_of_rows():
    x = np.array([[0.0, 0.0, 0.0], [448.0, -1.0, 2.0 ** -9], [449.0, 0.0, 1.0], [3.5, -3.5, 0.0], [2.0 ** -140, 0.0, 0.0],
                  [np.nan, 1.0, 2.0], [1.0, -np.inf, 2.0], [3.3e38, 1.0, -3.3e38]])
    codes, byte = ref.q8_rows(x)
    assert byte.tolist() == [127, 127, 128, 120, 0, 255, 255, 247]
    v = ref.q8_values(codes, byte)
    assert np.isnan(v[5:7]).all() and (codes[5:7] == 0).all()
    assert v[0].tolist() == [0, 0, 0] and v[1].tolist() == [448.0, -1.0, 2.0 ** -9] and v[3].tolist() == [3.5, -3.5, 0.0]
    assert v[7].tolist() == [240 * 2.0 ** 120, 0.0, -240 * 2.0 ** 120] and np.isfinite(np.float32(v[7])).all()
    assert v[2].tolist() == [448.0, 0.0, 1.0] and v[4, 0] in (0.0, 2.0 ** -136)
    r = np.random.default_rng(1).standard_normal((200, 64)) * np.exp(np.random.default_rng(2).standard_normal((200, 1)) * 5)
    codes, byte = ref.q8_rows(r)
    got, top = ref.q8_values(codes, byte), np.abs(r).max(-1, keepdims=True)
    assert (np.abs(got - r) <= np.maximum(np.abs(r) * 2.0 ** -4, top * 2.0 ** -10 / 224)).all()
    old, scale, deq = fp8.quantise_rows(r.astype(np.float32))
    codes, byte = ref.q8_rows(r.astype(np.float32))
    assert np.array_equal(old, codes) and np.array_equal(scale, 2.0 ** (byte.astype(np.float64) - 127))
    assert np.isnan(ref.q8_values(np.array([[0x7F, 0xFF, 0x7E]], np.uint8), np.array([127], np.uint8))).tolist() == [[True, True, False]]


def test_joining_is_attention_over_both_sets():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((5, 2, 8)), rng.standard_normal((1, 1, 20, 8)), rng.standard_normal((1, 1, 20, 8))
    start, table = [0, 5], np.zeros((1, 1), np.int64)
    o1, l1, _, _ = ref.attention(q, k, v, start, [15], table, 20, ref.PREFIX)
    own = np.swapaxes(k[0, :, 15:], 0, 1), np.swapaxes(v[0, :, 15:], 0, 1)
    o2, l2, _, _ = ref.packed(q, *own, start, ref.CAUSAL)
    o, l = ref.join(o1, l1, o2, l2)
    w, lw, _, _ = ref.attention(q, k, v, start, [15], table, 20, ref.CAUSAL)
    assert np.allclose(o, w, atol=1e-13) and np.allclose(l, lw, atol=1e-13)
    none = np.full_like(l1, -np.inf)
    o, l = ref.join(np.full_like(o1, np.nan), none, o2, l2)
    assert np.array_equal(o, o2) and np.array_equal(l, l2)
    o, l = ref.join(o1, none, o2, none)
    assert (o == 0).all() and np.isneginf(l).all()


def test_packed_rows_see_their_own_sequence():
    rng = np.random.default_rng(4)
    q, k, v = (rng.standard_normal((9, 1, 4)) for _ in range(3))
    o, l, _, _ = ref.packed(q, k, v, [0, 1, 1, 5], ref.CAUSAL)
    assert np.allclose(o[0], v[0]) and np.allclose(l[0, 0], q[0, 0] @ k[0, 0] / 2)       # alone: its own value
    assert (o[5:] == 0).all()                                                            # rows of no sequence
    a = np.exp(np.array([q[2, 0] @ k[1, 0], q[2, 0] @ k[2, 0]]) / 2)
    assert np.allclose(o[2, 0], (a[0] * v[1, 0] + a[1] * v[2, 0]) / a.sum())
    o1, _, _, _ = ref.packed(q, k, v, [0, 1, 1, 5], ref.BLOCK, window=1)
    assert not np.allclose(o1[2], v[2])                                                  # later rows are seen
    o2, _, _, _ = ref.packed(q, k, v, [0, 1, 1, 5], ref.CAUSAL, window=1)
    assert np.allclose(o2[:5], v[:5])
