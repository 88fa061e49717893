"""The token inputs of the attention's GPU tests, on the CPU: mistakes planted in
the definition (a token left out, taken twice, another token's value, 16 tokens of
the neighbouring 16) are outside the tolerance that those tests allow."""

import numpy as np
import pytest

import kv_ref as R
import kv_tokens as T


def half_step(x):
    """The farthest that rounding to bf16 can bring x towards what a test compares with."""
    return 2.0 ** -8 * np.abs(x)


def passes_counting(o, lse, wrong, wrong_lse):
    """Whether the test could pass, with the roundings of the wrong result as they suit it best."""
    return (np.abs(wrong - o) <= T.count_tolerance(o) + half_step(wrong)).all() and \
        abs(wrong_lse - lse) <= T.count_lse_tolerance(lse) * 2


@pytest.mark.parametrize("D,n", [(128, 9000), (128, 14000), (64, 7000), (128, 300), (64, 65)])
def test_every_token_counts(D, n):
    rng = np.random.default_rng(n)
    v = T.counting_values(n, 2, D, rng)
    assert (v.sum(2) == 1).all() and v.sum(0).max() <= -(-n // D)
    o, lse = T.counted(v, n - 1)
    assert np.allclose(o.sum(1), 1.0) and passes_counting(o, lse, o, lse)
    total = v.sum(0, dtype=np.float64)
    for t in rng.integers(0, n, 200):
        gone = (total - v[t]) / (n - 1), np.log(n - 1)
        twice = (total + v[t]) / (n + 1), np.log(n + 1)
        assert not passes_counting(o, lse, *gone) and not passes_counting(o, lse, *twice)
        u = (t + int(rng.choice([1, 16, 32, 64, 128, 1024]))) % n
        if (v[t] != v[u]).any():                            # another token's value: its columns change by one each
            assert not passes_counting(o, lse, (total - v[t] + v[u]) / n, lse), (t, u)
        g = t // 16 * 16
        if g + 32 <= n:                                     # 16 tokens of the neighbouring 16's values
            moved = (total - v[g:g + 16].sum(0) + v[g + 16:g + 32].sum(0)) / n
            assert not passes_counting(o, lse, moved, lse)
        if t >= 1:                                          # a row that sees one token less, or a window that does
            assert not passes_counting(*T.counted(v[:t + 1], t), *T.counted(v[:t + 1], t - 1))
            assert not passes_counting(*T.counted(v, n - 1, 1 + t, 0), *T.counted(v, n - 1, t, 0))


def test_counting_is_the_definition():
    rng = np.random.default_rng(0)
    v = T.counting_values(90, 2, 64, rng)
    pool = v.reshape(3, 30, 2, 64).transpose(0, 2, 1, 3).astype(np.float64)
    q = np.zeros((4, 4, 64))
    for window, sinks in ((0, 0), (20, 3), (1, 0)):
        o, lse, _, _ = R.attention(q, rng.standard_normal(pool.shape), pool, [0, 4], [85], np.array([[0, 1, 2]]), 0.1,
                                   window, sinks)
        for i in range(4):
            want, l = T.counted(v[:85], 81 + i, window, sinks)
            assert np.allclose(o[i], want.repeat(2, 0)) and np.allclose(lse[i], l)


@pytest.mark.parametrize("D", [64, 128])
def test_targets_take_the_weight(D):
    """Row by row the definition gives the target's value, and without the target, or with its neighbour's value, another
    row of values far beyond the tolerance."""
    rng = np.random.default_rng(D)
    n, heads, hq, page = 5000, 2, 8, 50
    k, v = rng.standard_normal((2, n, heads, D)).astype(np.float32)
    pos = np.arange(n - 9, n)
    q = rng.standard_normal((9, hq, D)).astype(np.float32)
    q = R.bf16(q).float().numpy()
    at = T.pick_targets(pos, heads, hq, rng)
    assert (at >= 0).all() and (at <= pos[:, None]).all()
    assert all(len(set(at[:, h * 4:h * 4 + 4].ravel())) == 36 for h in range(heads))
    T.aim(k, q, at)
    for fmt in ("bf16", "mx"):
        kq, vq = ((R.bf16(x).double().numpy() if fmt == "bf16" else R.mx_values(*R.mx_quantize(x))) for x in (k, v))
        kp, vp = (x.reshape(-1, page, heads, D).transpose(0, 2, 1, 3) for x in (kq, vq))
        scale = float(np.float32(D ** -0.5))
        o, lse, mag, size = R.attention(q.astype(np.float64), kp, vp, [0, 9], [n], np.arange(100)[None], scale)
        tol = R.tolerance(o, mag, size, D, scale, n, np.abs(vp).max())
        target = vq[at, np.arange(hq) // 4]
        assert (np.abs(o - target) < 1e-4).all()
        assert (tol <= 2.0 ** -6 * np.abs(target) + 1e-4).all()
        for step in (-1, 1, 16, -64):                       # another token's value
            other = vq[(at + step) % n, np.arange(hq) // 4]
            assert (np.abs(other - o) > tol).any(-1).all()
