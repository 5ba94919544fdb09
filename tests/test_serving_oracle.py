"""The plain definitions of head norms, rotation, page forks and compaction on cases that can be checked by hand."""
import numpy as np

from oracle import paged_oracle as P
from oracle import serving_oracle as S


def test_norm_and_rotation_by_hand():
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])
    assert np.allclose(S.normed(x, np.array([1.0, 2.0, 1.0, 1.0]), 0.0), [[[3 / 2.5, 8 / 2.5, 0, 0]]])
    assert np.array_equal(S.normed(x, None, 1.0), x)
    quarter = np.array([np.pi / 2, 0.0])
    assert np.allclose(S.turned(x, [1], quarter, False), [[[0.0, 4.0, 3.0, 0.0]]])       # pairs (0, 2) and (1, 3)
    assert np.allclose(S.turned(x, [1], quarter, True), [[[-4.0, 3.0, 0.0, 0.0]]])       # pairs (0, 1) and (2, 3)
    # a score depends on the distance alone
    rng = np.random.default_rng(0)
    q, k, f = rng.normal(size=(1, 1, 8)), rng.normal(size=(1, 1, 8)), np.array([1.0, 0.3, 0.01])
    for near in (False, True):
        a = (S.turned(q, [107], f, near) * S.turned(k, [100], f, near)).sum()
        b = (S.turned(q, [7], f, near) * S.turned(k, [0], f, near)).sum()
        assert abs(a - b) < 1e-12


def test_fork_by_hand():
    """Two sequences that share page 5: the second is replaced by the first, the third is done."""
    o = P.Pages([[5, 1, -1], [5, 2, -1], [7, -1, -1]], [100, 70, 64], [0, 3, 4, 6, -9, -9, -9, -9], 4, 8)
    shares = [0, 0, 0, 0, 0, 1, 0, 0]
    copies, short = S.fork(o, shares, [0, 0, -1], [100, 100, 9])
    assert not short and copies == [(1, 2, 36)]              # page 2 and 7 went back; the lowest is taken first
    assert o.table == [[5, 1, -1], [5, 2, -1], [-1, -1, -1]] and o.kv_len == [100, 100, 0]
    assert o.free[:o.n_free] == [0, 3, 4, 6, 7] and shares == [0, 0, 0, 0, 0, 1, 0, 0]
    # a page that another sequence has in full is copied by all that have less of it
    o = P.Pages([[5, -1], [-1, -1], [-1, -1]], [64, 0, 0], [0, 1, 2, -9, -9, -9], 3, 6)
    shares = [0] * 6
    copies, short = S.fork(o, shares, [0, 0, 0], [64, 10, 20])
    assert not short and copies == [(5, 2, 10), (5, 1, 20)] and shares == [0] * 6 and o.table == [[5, -1], [2, -1], [1, -1]]


def test_compact_by_hand():
    o = P.Pages([[6, 1], [4, -1]], [100, 3], [5, 0, 2, 3, -9, -9, -9], 4, 7)
    shares = [0, 0, 0, 0, 0, 0, 1]
    assert S.compact(o, shares, 9) == [(6, 0, 64), (4, 2, 64)]
    assert o.table == [[0, 1], [2, -1]] and o.free[:4] == [6, 5, 4, 3] and shares == [1, 0, 0, 0, 0, 0, 0]
    assert S.compact(o, shares, 9) == []


def test_cross_by_hand():
    q, k, v = np.ones((1, 2, 1)), np.array([[[0.0]], [[np.log(3.0)]]]), np.array([[[4.0]], [[-8.0]]])
    out, mag = S.cross(q, k, v, 1.0)
    assert np.allclose(out, -5.0) and np.allclose(mag, 7.0)
    assert not S.cross(q, k[:0], v[:0], 1.0)[0].any()
