"""Pins of the paged-cache oracle: closed forms, hand-worked slots, textbook softmax."""
import numpy as np

from oracle import paged


def test_rotation_closed_forms():
    x = np.random.default_rng(0).standard_normal((5, 2, 8))
    pos = np.arange(5)
    assert np.array_equal(paged.rotate(x, pos, []), x)
    assert np.allclose(paged.rotate(x, 0 * pos, [1.0, 0.5]), x, atol=0)            # position 0 turns nothing
    quarter = paged.rotate(x, pos * 0 + 1, [np.pi / 2, np.pi])                      # a quarter and a half turn
    assert np.allclose(quarter[..., 0], -x[..., 2]) and np.allclose(quarter[..., 2], x[..., 0])
    assert np.allclose(quarter[..., 1], -x[..., 1]) and np.allclose(quarter[..., 3], -x[..., 3])
    assert np.array_equal(quarter[..., 4:], x[..., 4:])
    inter = paged.rotate(x, pos * 0 + 1, [np.pi / 2, np.pi], interleaved=True)
    assert np.allclose(inter[..., 0], -x[..., 1]) and np.allclose(inter[..., 1], x[..., 0])
    assert np.allclose(inter[..., 2], -x[..., 2]) and np.allclose(inter[..., 3], -x[..., 3])


def test_rotation_keeps_lengths_and_makes_products_relative():
    rng = np.random.default_rng(1)
    q, k, f = rng.standard_normal((1, 1, 8)), rng.standard_normal((1, 1, 8)), [1.0, 0.3, 0.01, 0.001]
    for inter in (False, True):
        at = lambda x, p: paged.rotate(x, np.array([p]), f, inter)
        assert np.isclose(np.linalg.norm(at(q, 1234)), np.linalg.norm(q))
        assert np.isclose((at(q, 1007) * at(k, 1000)).sum(), (at(q, 7) * at(k, 0)).sum())


def test_slots_by_hand():
    table = [4, -1, 2]
    assert paged.slots(6, 6, table, 8, 5) == [(4, 6), (4, 7), (-1, 0), (-1, 1), (-1, 2), (-1, 3)]
    assert paged.slots(22, 3, table, 8, 5) == [(2, 6), (2, 7), (-1, 0)]             # behind the table
    assert paged.slots(-1, 2, table, 8, 5) == [(-1, 7), (4, 0)]
    assert paged.slots(0, 1, table, 8, 4) == [(-1, 0)]                               # page 4 of a pool of 4


def test_ordered_rows_and_attention():
    rng = np.random.default_rng(2)
    pool = rng.standard_normal((5, 8, 2, 4))
    dense = paged.ordered(pool, [3, 0], 11)
    assert np.array_equal(dense, np.concatenate([pool[3], pool[0][:3]]))
    q = rng.standard_normal((6, 4))
    out, lse = paged.token_attention(q, dense, dense + 1, 0.5)
    for h in range(6):
        s = 0.5 * dense[:, h // 3] @ q[h]
        assert np.allclose(out[h], (np.exp(s) / np.exp(s).sum()) @ (dense[:, h // 3] + 1)) and np.isclose(lse[h], np.log(np.exp(s).sum()))
    out, lse = paged.token_attention(q, dense[:1], dense[:1], 0.5)                   # one key: its value
    assert np.allclose(out, np.repeat(dense[0], 3, 0))
    out, lse = paged.token_attention(q, dense[:0], dense[:0], 0.5)
    assert not out.any() and np.isneginf(lse).all()
