"""Pins of the key/value cache's oracle: hand-worked assignments, the 8-bit
type's table, and attention against a dense softmax."""
import numpy as np

from oracle import kv_cache as kv


def test_assignment_by_hand():
    # Blocks of 8.  Request 0: 5 cached, 4 new: fills its block (3 places), opens one.  Request 1: a fresh prompt of 17:
    # three blocks.  Request 2: 16 cached, 1 new: its two blocks are full, opens one.  Request 3: 3 cached, 2 new: none.
    table = np.full((4, 4), -1)
    table[0, 0], table[2, :2], table[3, 0] = 7, (2, 9), 4
    t, start, seq, pos, slots, counts = kv.assign([5, 0, 16, 3], [4, 17, 1, 2], table, [10, 11, 12, 13, 14, 15], 8, 26)
    assert start.tolist() == [0, 4, 21, 22, 24]
    assert seq.tolist() == [9, 17, 17, 5]
    assert t.tolist() == [[7, 10, -1, -1], [11, 12, 13, -1], [2, 9, 14, -1], [4, -1, -1, -1]]
    assert pos.tolist() == [5, 6, 7, 8] + list(range(17)) + [16, 3, 4, -1, -1]
    assert slots.tolist() == ([61, 62, 63, 80] + list(range(88, 96)) + list(range(96, 104)) + [104, 112, 35, 36, -1, -1])
    assert counts.tolist() == [24, 4, 5, 5]


def test_assignment_refuses_in_order():
    table = np.full((5, 2), -1)
    table[3, 0] = 1
    # free blocks: 2.  0 takes one; 1 would need 3 columns: refused without asking; 2 asks for two, one is left: refused,
    # and what it asked for is gone; 3 needs none: admitted; 4 asks for one past the end: refused.
    t, start, seq, pos, slots, counts = kv.assign([0, 0, 0, 2, 0], [8, 17, 9, 3, 1], table, [5, 6], 8, 100)
    assert seq.tolist() == [8, 0, 0, 5, 0]
    assert counts.tolist() == [38, 2, 1, 4]
    assert t.tolist() == [[5, -1], [-1, -1], [-1, -1], [1, -1], [-1, -1]]
    assert (pos[8:34] == -1).all() and pos[34:37].tolist() == [2, 3, 4] and (pos[37:] == -1).all()


def test_assignment_stops_at_the_token_limit():
    t, start, seq, pos, slots, counts = kv.assign([0, 0, 0], [4, 5, 1], np.full((3, 4), -1), list(range(9)), 8, 9)
    assert seq.tolist() == [4, 5, 0] and start.tolist() == [0, 4, 9, 10] and counts.tolist() == [10, 2, 2, 2]


def test_e4m3_by_hand():
    x = [0.0, 1.0, 1.0625, 1.1875, 1.125, 17.0, 19.0, 448.0, 464.0, 1e9, -1e9, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 0.015625]
    want = [0.0, 1.0, 1.0, 1.25, 1.125, 16.0, 20.0, 448.0, 448.0, 448.0, -448.0, 2.0 ** -9, 0.0, 2.0 ** -8, 0.015625]
    assert kv.round_e4m3(x).tolist() == want
    assert np.isnan(kv.round_e4m3(np.nan)) and kv.round_e4m3(-np.inf) == -448.0


def test_e4m3_agrees_with_the_type():
    import torch
    x = np.concatenate([np.linspace(-460, 460, 4001), np.exp2(np.linspace(-12, 9, 999))]).astype(np.float32)
    ref = torch.tensor(x).clamp(-448, 448).to(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(kv.round_e4m3(x), ref)


def test_attention_is_a_causal_softmax():
    rng = np.random.default_rng(3)
    heads, kv_heads, d, bs, length, new = 6, 2, 16, 8, 21, 5
    k, v = rng.standard_normal((2, length, kv_heads, d))
    q = rng.standard_normal((new, heads, d))
    table = np.array([[2, 0, 3]])
    kc, vc = rng.standard_normal((2, 4, kv_heads, bs, d))
    for c, x in ((kc, k), (vc, v)):
        for p in range(length):
            c[table[0, p // bs], :, p % bs] = x[p]
    for window in (0, 4):
        out, spread, _ = kv.attention(q, kc, vc, table, [0, new], [length], 0.3, window)
        for j in range(new):
            p = length - new + j
            lo = 0 if not window else p - window + 1
            for h in range(heads):
                g = h // 3
                w = np.exp(0.3 * (k[lo:p + 1, g] @ q[j, h]))
                np.testing.assert_allclose(out[j, h], (w / w.sum()) @ v[lo:p + 1, g], rtol=1e-12, atol=1e-13)
                assert (spread[j, h] >= np.abs(out[j, h]) - 1e-12).all()


def test_attention_of_rows_that_see_nothing():
    rng = np.random.default_rng(4)
    q, kc, vc = rng.standard_normal((4, 2, 8)), rng.standard_normal((2, 1, 8, 8)), rng.standard_normal((2, 1, 8, 8))
    # request 0 is empty; request 1 holds one position for two queries; row 3 is nobody's
    out, _, _ = kv.attention(q, kc, vc, np.array([[0], [1]]), [0, 1, 3], [0, 1], 1.0)
    assert (out[:2] == 0).all() and np.array_equal(out[2, 0], vc[1, 0, 0]) and np.isnan(out[3]).all()
