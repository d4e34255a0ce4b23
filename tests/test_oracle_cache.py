"""What pins the context-cache oracle (oracle/cache.py): hand-made cases, closed
forms, and the unwindowed oracle."""

import numpy as np
import pytest

from oracle import attention as OT
from oracle import cache as OC


def test_window_by_hand():
    # six context slots, a chain 0 <- 1 <- 2 at positions 6, 7, 8, window 3, one sink
    vis = OC.visible(6, 3, [-1, 0, 1], n_sinks=1, window=3)
    assert vis[0].nonzero()[0].tolist() == [0, 4, 5, 6]
    assert vis[1].nonzero()[0].tolist() == [0, 5, 6, 7]
    assert vis[2].nonzero()[0].tolist() == [0, 6, 7, 8]
    # siblings do not see each other; a window of one leaves the row itself
    vis = OC.visible(2, 3, [-1, 0, 0], window=1)
    assert [r.nonzero()[0].tolist() for r in vis] == [[2], [3], [4]]
    # a sink among the new keys stays visible
    vis = OC.visible(0, 4, [-1, 0, 1, 2], n_sinks=1, window=2)
    assert vis[3].nonzero()[0].tolist() == [0, 2, 3]
    # a block's rows see the whole block
    assert OC.visible(5, 2, None, window=2).astype(int).tolist() == [[0, 0, 0, 0, 1, 1, 1], [0, 0, 0, 0, 0, 1, 1]]


def test_window_as_wide_as_the_context_is_none():
    rng = np.random.default_rng(0)
    q, kn, vn = rng.normal(size=(1, 5, 4, 32)), rng.normal(size=(1, 5, 2, 32)), rng.normal(size=(1, 5, 2, 32))
    k, v = rng.normal(size=(1, 2, 40, 32)), rng.normal(size=(1, 2, 40, 32))
    par = [[-1, 0, 0, 1, 3]]
    want = OT.tree_verify_attn(q, k, v, kn, vn, [40], par)
    for window, sinks in ((0, 0), (44, 0), (1, 45)):
        got = OC.attention(q, k, v, kn, vn, [40], par, sinks, window)
        np.testing.assert_allclose(got[0], want[0], rtol=1e-12)
        np.testing.assert_allclose(got[1], want[1], rtol=1e-12)


def test_sliding_window_is_local_causal_attention():
    """A chain verified over a windowed context equals banded causal attention over the whole sequence."""
    rng = np.random.default_rng(1)
    total, ctx, w = 30, 22, 6
    q, k, v = (rng.normal(size=(total, 1, 8)) for _ in range(3))
    got, _ = OC.attention(q[None, ctx:], k[None, :ctx].transpose(0, 2, 1, 3), v[None, :ctx].transpose(0, 2, 1, 3), k[None, ctx:],
                          v[None, ctx:], [ctx], [list(range(-1, total - ctx - 1))], 0, w)
    s = q[:, 0] @ k[:, 0].T / np.sqrt(8)
    i, j = np.indices(s.shape)
    s = np.where((j <= i) & (i - j < w), s, -np.inf)
    p = np.exp(s - s.max(1, keepdims=True))
    want = (p / p.sum(1, keepdims=True)) @ v[:, 0]
    np.testing.assert_allclose(got[0, :, 0], want[ctx:], rtol=1e-12)


def _block(*values):
    x = np.zeros(32)
    x[:len(values)] = values
    return x


@pytest.mark.parametrize("largest,exp", [(6.0, 0), (6.99, 0), (7.0, 1), (8.0, 1), (4.0, 0), (3.5, 0), (3.49, -1), (2 ** -125.0, -125),
                                         (2.0 ** -149, -125), (0.0, -125), (3.0e38, 125), (1.0e38, 124), (1.75, -1), (1.7499, -2)])
def test_block_exponent(largest, exp):
    # the largest magnitude, rounded to two significant bits, lies two powers above 2^e
    assert OC.block_exponent(_block(-largest)) == exp


def test_rounding_to_codes():
    x = _block(0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.26, 5.01, -5.0, -0.0, 6.9, 6.0, -0.24)
    codes, scales = OC.encode(x)
    assert scales.tolist() == [127]
    assert codes[:14].tolist() == [0, 2, 2, 4, 4, 6, 6, 1, 7, 14, 8, 7, 7, 8]
    back = OC.decode(OC.pack(codes), scales)
    assert back[:4].tolist() == [0.0, 1.0, 1.0, 2.0] and back[9] == -4.0
    # values on the grid come back as they are
    again, s2 = OC.encode(back)
    np.testing.assert_array_equal(OC.decode(OC.pack(again), s2), back)


def test_non_finite_blocks_read_nan():
    for bad in (np.nan, np.inf, -np.inf):
        codes, scales = OC.encode(np.concatenate([_block(1.0, bad), _block(2.0)]))
        assert scales[0] == 255 and scales[1] != 255
        back = OC.decode(OC.pack(codes), scales)
        assert np.isnan(back[:32]).all() and back[32] == 2.0


def test_quantisation_error_is_bounded():
    rng = np.random.default_rng(2)
    x = rng.normal(size=(64, 128)) * np.exp(rng.normal(size=(64, 1)) * 4)
    codes, scales = OC.encode(x)
    back = OC.decode(OC.pack(codes), scales)
    unit = 2.0 ** np.repeat(scales.astype(float) - 127, 32, axis=-1)
    # half a step, a step being at most 2 units in [4, 6]; what is clipped loses less than one unit
    assert (np.abs(back - x) <= unit).all()
    assert (np.abs(x) < 7 * unit).all()


def test_weights_of_a_whole_block_sum_to_the_rows():
    """Every row's attention sums to one over context and new keys."""
    rng = np.random.default_rng(3)
    q, kn, vn = rng.normal(size=(1, 3, 4, 32)), rng.normal(size=(1, 3, 2, 32)), rng.normal(size=(1, 3, 2, 32))
    k, v = rng.normal(size=(1, 2, 20, 32)), rng.normal(size=(1, 2, 20, 32))
    _, lse = OC.attention(q, k, v, kn, vn, [17], [[-1, 0, 1]])
    old = rng.random((1, 2, 20))
    got = OC.weigh(q, k, lse, [17], old, 0.5, kn, [2], [[0, 1, 2, -1]])
    fresh = got - np.where(np.arange(20) < 17, 0.5 * old, 0.0)
    np.testing.assert_allclose(fresh.sum(-1), 3 * 2, rtol=1e-12)  # three rows, two query heads a KV head
    # a path that ends early counts fewer rows, and slots behind it keep their weight
    got = OC.weigh(q, k, lse, [17], old, 1.0, kn, [2], [[0, 5, 2, -1]])
    np.testing.assert_array_equal(got[..., 18:], old[..., 18:])
    got = OC.weigh(q, k, lse, [17], old, 0.25, kn, [-1], [[-1, -1, -1, -1]])
    np.testing.assert_allclose(got[..., :17], 0.25 * old[..., :17])


def test_evict_by_hand():
    w = np.array([[[5.0, 0.0, 3.0, 3.0, np.nan, 3.0, 1.0, 0.0]]])
    assert OC.evict([8], w, 8)[0][0] == list(range(8))
    assert OC.evict([8], w, 4)[0][0] == [0, 2, 3, 4]              # ties: the lowest slots
    assert OC.evict([8], w, 4, n_sinks=2, n_recent=1)[0][0] == [0, 1, 4, 7]
    assert OC.evict([3], w, 4)[0][0] == [0, 1, 2]
    assert OC.evict([8], w, 3, n_sinks=1, n_recent=2)[0][0] == [0, 6, 7]
