"""The oracle of the operators around the loss pass, against what can be said without it."""

import numpy as np

from oracle import operators_oracle as oo


def test_blocks_take_the_nearest_value_and_even_codes_at_ties():
    x = np.zeros((1, 40))
    x[0, :32] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, 5.01, 7.9, 0.26, 0.24, -6.1, 0.0] + 16 * [1.0]
    codes, exps, values = oo.mx4_blocks(x)
    assert list(values[0, :16]) == [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 0.0, -1.0, 6.0, 6.0, 0.5, 0.0, -6.0, 0.0]
    assert exps[0, 0] == 127 and exps[0, 1] == 0 and (values[0, 32:] == 0).all()
    for scale in (2.0 ** -100, 2.0 ** 90):
        assert (oo.mx4_blocks(x * scale)[2] == values * scale).all()
    again = oo.mx4_blocks(values)[2]
    assert (again == values).all()                                   # what is held is held again
    bad = x.copy()
    bad[0, 3] = np.inf
    assert np.isnan(oo.mx4_blocks(bad)[2][0, :32]).all() and oo.mx4_blocks(bad)[1][0, 0] == 255


def test_packed_bytes_hold_every_scale_once():
    rng = np.random.RandomState(0)
    x = rng.randn(70, 300) * 2.0 ** rng.randint(-8, 8, (70, 1))
    packed = oo.mx4_packed(x).reshape(4, 8704)
    _, exps, _ = oo.mx4_blocks(x)
    assert sorted(b for b in packed[:, 8192:].reshape(-1) if b) == sorted(exps.reshape(-1).tolist())


def test_verified_tokens_have_the_targets_distribution():
    rng = np.random.RandomState(1)
    V, n = 5, 40000
    z, zq = rng.randn(1, V), rng.randn(1, V)
    p = np.exp(z[0]) / np.exp(z[0]).sum()
    q = np.exp(zq[0]) / np.exp(zq[0]).sum()
    for draft in (zq, None):
        seen = np.zeros(V)
        for _ in range(n // 4):
            x = rng.choice(V, p=q)
            rows = np.concatenate([z, z])
            got = oo.verify(rows, None if draft is None else np.concatenate([draft, draft]), [x, 0], [0], [1], [1.0],
                            rng.rand(2), rng.exponential(size=(1, V)))[0]
            seen[x if got["kept"] else got["token"]] += 1
        if draft is not None:                                        # (a looked-up draft that is drawn from q is biased)
            assert np.abs(seen / seen.sum() - p).max() < 5 * 0.5 / np.sqrt(n // 4)
        else:
            kept_or_other = q * p + np.array([sum(q[x] * (1 - p[x]) * p[v] / (1 - p[x]) for x in range(V) if x != v) for v in range(V)])
            assert np.abs(seen / seen.sum() - kept_or_other).max() < 5 * 0.5 / np.sqrt(n // 4)


def test_identical_distributions_keep_everything_and_greedy_follows_the_largest():
    rng = np.random.RandomState(2)
    z = rng.randn(4, 9)
    ids = rng.randint(0, 9, 4)
    got = oo.verify(z, z, ids, [0], [3], [0.7], [0.9999, 0.5, 0.0, 0.0], rng.exponential(size=(1, 9)))[0]
    assert got["kept"] == 3
    best = z.argmax(axis=1)
    got = oo.verify(z, z, [best[0], best[1], (best[2] + 1) % 9, 0], [0], [3], [0.0], np.zeros(4), rng.exponential(size=(1, 9)))[0]
    assert got["kept"] == 2 and got["token"] == best[2]


def test_clipping_by_differences():
    grads = [np.array([3.0, 4.0]), np.array([12.0])]
    total, norm, c, outs = oo.grad_clip(grads, 6.5, 0.0)
    assert total == 169 and norm == 13 and c == 0.5 and outs[1][0] == 6.0
    assert oo.grad_clip(grads, 20.0, 0.0)[2] == 1.0
