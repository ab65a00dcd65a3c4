"""The 8-bit cache's reference pinned on the CPU: e4m3 codes, scales, re-rounding, bounds, selection."""
import numpy as np
import pytest

import oracle.qcache as Q


def _empty(pages=4, H=1, D=8, table=((0, 1, 2, 3),)):
    z = np.zeros
    return Q.Cache(z((pages, H, 64, D), np.uint8), z((pages, H, 16, D, 4), np.uint8), z((pages, H), np.int64),
                   z((pages, H), np.int64), z((pages, H, 2, D), np.int64), np.asarray(table, np.int32))


def test_codes_match_the_format():
    import torch
    codes = np.arange(256, dtype=np.uint8)
    ref = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(ref, nan=7e7), np.nan_to_num(Q.VALUES, nan=7e7))
    fin = codes[(codes & 127) != 127]
    assert np.array_equal(Q.encode(Q.VALUES[fin]) & 127, fin & 127)
    x = np.random.default_rng(0).normal(size=20000) * np.exp2(np.random.default_rng(1).integers(-12, 7, 20000))
    mid = (Q.VALUES[:126] + Q.VALUES[1:127]) / 2
    x = np.clip(np.concatenate([x, mid, -mid]), -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(Q.encode(x), want)


@pytest.mark.parametrize("a,e", [(0.0, -32), (448.0, 0), (448.0001, 1), (224.0, -1), (65504.0, 8), (1e-30, -32), (3.5, -7)])
def test_scale_exponent(a, e):
    assert Q.scale_exponent(a) == e


def test_older_codes_move_to_a_larger_scale():
    c = _empty()
    rng = np.random.default_rng(2)
    small, large = rng.normal(size=(5, 1, 8)), 300 * rng.normal(size=(3, 1, 8))
    Q.append(c, 0, 0, small, small)
    before = Q.VALUES[c.k[0, 0, :5]] * 2.0 ** c.ke[0, 0]
    Q.append(c, 0, 5, large, large)
    after = Q.VALUES[c.k[0, 0, :5]] * 2.0 ** c.ke[0, 0]
    assert c.ke[0, 0] == Q.scale_exponent(np.abs(large).max())
    # exact where the value stays normal, half a subnormal step otherwise
    assert np.all(np.abs(after - before) <= 2.0 ** (c.ke[0, 0] - 10))
    hi, lo = c.bounds[0, 0] * 4 * 2.0 ** c.ke[0, 0]
    K = Q.VALUES[c.k[0, 0, :8]] * 2.0 ** c.ke[0, 0]
    assert np.all(K <= hi) and np.all(K >= lo)


def test_bounds_hold_over_many_appends():
    c = _empty()
    rng = np.random.default_rng(3)
    p = 0
    for n in (1, 3, 1, 30, 2, 64, 40):
        x = rng.normal(size=(n, 1, 8)) * np.exp2(rng.integers(-6, 6))
        Q.append(c, 0, p, x, x)
        p += n
    for lp in range(-(-p // 64)):
        n = min(64, p - 64 * lp)
        K = Q.VALUES[c.k[lp, 0, :n]]
        assert np.all(K <= 4 * c.bounds[lp, 0, 0]) and np.all(K >= 4 * c.bounds[lp, 0, 1])


def test_bounds_of_a_page_that_began_with_nan():
    """NaN tokens leave no bounds behind, whatever the scale does afterwards."""
    c = _empty()
    x = np.full((2, 1, 8), 0.25)
    x[:, 0, :3] = np.nan
    Q.append(c, 0, 0, x, x)
    assert c.bounds[0, 0, :, 0].tolist() == [-128, 127]
    y = -np.abs(np.random.default_rng(8).normal(size=(3, 1, 8)) * 300) - 1000
    Q.append(c, 0, 2, y, y)
    K = Q.VALUES[c.k[0, 0, :5]]
    assert np.array_equal(c.bounds[0, 0, 0], np.ceil(np.nanmax(K, 0) / 4))
    assert np.array_equal(c.bounds[0, 0, 1], np.floor(np.nanmin(K, 0) / 4))


def test_what_dropped_positions_leave_behind():
    """A page whose open end is written again and again by positions that are dropped: committed codes are off by less than
    a subnormal step (2^-9) of the scale that was reached, for all growths together, and the bounds still hold."""
    rng = np.random.default_rng(9)
    kept, used = _empty(), _empty()
    for first in range(0, 60, 3):
        x = rng.normal(size=(3, 1, 8)) * np.exp2(rng.integers(-12, 1))
        Q.append(kept, 0, first, x, x)
        Q.append(used, 0, first, x, x)
        scratch = rng.normal(size=(4, 1, 8)) * 2.0 ** (first / 5)  # larger every time
        Q.append(used, 0, first + 3, scratch, scratch)
    e = int(used.ke[0, 0])
    assert e >= kept.ke[0, 0] + 8 and e == used.ve[0, 0]
    for a, b in ((kept.k, used.k), (kept.v.transpose(0, 1, 2, 4, 3).reshape(kept.k.shape), used.v.transpose(0, 1, 2, 4, 3).reshape(kept.k.shape))):
        a, b = (Q.VALUES[x[0, 0, :60]] * 2.0 ** s for x, s in ((a, int(kept.ke[0, 0])), (b, e)))
        # (a growth by g >= 1 exponents rounds to half a step of the new scale: 1/2 + 1/4 + ... of the last one's step, and
        # once where the token itself was rounded at either scale, by half a step or 2^-4 of it)
        assert np.all(np.abs(a - b) <= 2.0 ** (e - 9) + 2.0 ** -3 * np.abs(a))
    K = Q.VALUES[used.k[0, 0, :60]]
    assert np.all(K <= 4 * used.bounds[0, 0, 0]) and np.all(K >= 4 * used.bounds[0, 0, 1])


def test_nan_reaches_those_who_see_it_only():
    c = _empty()
    x = np.random.default_rng(4).normal(size=(10, 1, 8))
    v = x.copy()
    v[6, 0, 3] = np.nan
    Q.append(c, 0, 0, x, v)
    q = np.ones((1, 8))
    assert np.all(np.isfinite(Q.attend(c, 0, 0, q, 6, 0.3)[0])) and np.all(np.isnan(Q.attend(c, 0, 0, q, 7, 0.3)[0]))
    assert not np.isnan(Q.VALUES[c.v]).any()


def test_selection_ranks_by_the_bound_and_keeps_the_newest():
    c = _empty()
    rng = np.random.default_rng(5)
    x = rng.normal(size=(200, 1, 8))
    x[64:128] += 5
    Q.append(c, 0, 0, x, x)
    assert Q.select(c, 0, 0, np.ones((1, 8)), 200, 2) == [1, 3]
    assert Q.select(c, 0, 0, np.zeros((1, 8)), 200, 2) == [0, 3]  # ties: the lowest
    assert Q.select(c, 0, 0, np.ones((1, 8)), 70, 2) == [0, 1]
    c.table[0, 1] = -1
    assert Q.select(c, 0, 0, np.ones((1, 8)), 200, 2)[-1] == 3 and 1 not in Q.select(c, 0, 0, np.ones((1, 8)), 200, 3)


def test_attention_of_the_whole_row_is_the_plain_softmax():
    c = _empty()
    x = np.random.default_rng(6).normal(size=(100, 1, 8))
    Q.append(c, 0, 0, x, 2 * x)
    K, V, _ = Q.keys_values(c, 0, 0, [0, 1])
    q = np.random.default_rng(7).normal(size=(3, 8))
    s = q @ K[:100].T * 0.5
    p = np.exp(s) / np.exp(s).sum(1, keepdims=True)
    assert np.allclose(Q.attend(c, 0, 0, q, 100, 0.5)[0], p @ V[:100], rtol=1e-12)
    assert np.array_equal(Q.attend(c, 0, 0, q, 0, 0.5)[0], np.zeros((3, 8)))
