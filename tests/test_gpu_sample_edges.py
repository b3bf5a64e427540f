"""GPU tests of the sampler where its sums, bins and cuts are at their edges, against the float64 model."""
import math

import numpy as np
import pytest

from tests import block_oracle as O
from tests.test_gpu_block_operators import _sample

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

FLT_MAX = float(np.finfo(np.float32).max)


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _lowest(f32):
    return float(torch.finfo(torch.float32 if f32 else torch.bfloat16).min)


def _check(x, f32=True, ld=None, shift=0, **par):
    got, lp, v = _sample(x, f32, ld, shift, **par)
    kinds = {k: np.int32 if k == "top_k" else np.float32 for k in par if par[k] is not None}
    cols = {k: np.broadcast_to(np.asarray(par[k], t), (len(v),)) for k, t in kinds.items()}
    for r in range(len(v)):
        p = {k: c[r].item() for k, c in cols.items()}
        token, want = O.sample(v[r], **p)
        assert got[r] == token, (r, p, got[r], token)
        # a weight and a sum of weights right to 2^-36 each, one rounding of the logarithm to fp32
        assert lp[r] == want or abs(lp[r] - want) <= 2.0**-24 * abs(want) + 2.0**-35, (r, p, lp[r], want)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("temperature", [1e35, 1e36, 1e37, 1e38, FLT_MAX])
def test_top_p_over_slices_of_the_lowest_value(temperature, f32):
    """Slices whose largest logit is far below -2^100, at temperatures at which that is no distance: their bins count
    from that logit.  Whole pieces only, and nothing that is not finite."""
    rng = np.random.default_rng([int(math.log10(temperature)), f32])
    n, low = 40960, _lowest(f32)
    x = rng.standard_normal((5, n))
    x[0, 8192:] = low                                        # all slices but the first
    x[1] = low
    x[2, :30000] = low * rng.uniform(0.5, 1.0, 30000)
    x[3] = np.clip(x[3] * 1e38, low, -low)
    x[4, ::2] = low
    for p in (0.3, 0.9, 0.9999):
        _check(x, f32, temperature=temperature, top_p=p, u=rng.random(5))


HOT = [1e28, 3.8e28, 1e29, 1e30, 1e37, FLT_MAX, math.inf]


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("temperature", HOT)
def test_top_p_leaves_out_what_has_no_mass_at_any_temperature(temperature, f32):
    """-inf, NaN and the places beside the row in its first and last piece: never part of the mass, however flat w is."""
    rng = np.random.default_rng([HOT.index(temperature), f32])
    for n, shift in ((100, 0), (1001, 3), (1001, 5), (8191, 1), (30011, 7), (140001, 2)):
        x = np.round(rng.standard_normal((6, n)) * 4) / 4
        x[0, n // 10:] = -np.inf
        x[1, rng.random(n) < 0.5] = -np.inf
        x[2, : n - n // 20] = np.nan
        x[3, rng.random(n) < 0.3] = np.nan
        x[4] = -np.inf
        x[4, [0, n // 2, n - 1]] = 1.0, 2.0, 3.0
        for p in (0.5, 0.9, 0.01):
            _check(x, f32, ld=n + 3, shift=shift, temperature=temperature, top_p=p, u=rng.random(6))
        _check(x, f32, ld=n + 3, shift=shift, temperature=temperature, top_p=0.7, min_p=0.5, u=0.0)


def test_top_p_of_masked_tokens_by_hand():
    """1000 tokens of which 500 are masked, weights alike to 2^-80: a nucleus of a half keeps 250."""
    x = np.full((1, 1000), -np.inf)
    x[0, ::2] = np.linspace(1, 0, 500)
    for t in (1e30, FLT_MAX):
        got, lp, _ = _sample(x, temperature=t, top_p=0.5, u=0.9999999)
        assert got[0] == 498 and lp[0] == np.float32(-math.log(250))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("value", [0.0, 1.0, 3.0, -1.0, -19.625, 7.25, 100.5, -1000.0])
def test_top_p_at_exact_ties(value, f32):
    """Equal logits alone have mass: the share that top_p asks for ends with a token exactly, which is the last one kept.
    In one slice and several, in lists, in a bin of its own (4000) and in more tokens than a list holds."""
    u = np.array([0.0, 0.25, 0.5, 0.75, 1 - 2.0**-24])
    for n, kept in ((20, 2), (20, 4), (1000, 100), (30000, 2), (30000, 100), (5000, 4000), (30000, 4000), (30000, 4096), (40000, 20000)):
        x = np.full((5, n), -np.inf)
        x[:, :: n // kept][:, :kept] = value
        assert (x[0] > -np.inf).sum() == kept
        for p in (0.25, 0.5, 0.75, np.float32(0.1)):
            for temperature in (1.0, 0.7):
                got, lp, _ = _sample(x, f32, temperature=temperature, top_p=p, u=u)
                count = math.ceil(float(np.float32(p)) * kept)
                assert got.tolist() == [n // kept * int(math.floor(a * count)) for a in u.astype(np.float32).astype(float)], (n, kept, p)
                assert (lp == np.float32(-math.log(count))).all(), (n, kept, p)


@pytest.mark.parametrize("f32", [False, True])
def test_top_p_does_not_change_with_the_rows_level(f32):
    """The same row some eighths higher or lower: the same draws, ties among its largest logits too."""
    rng = np.random.default_rng([16, f32])
    x = np.round(rng.standard_normal((8, 3000)) * 4) / 8
    x[:, rng.permutation(3000)[:40]] = 4.0
    x[4:] = np.where(x[4:] == 4.0, 4.0, -np.inf)
    u = rng.random(8)
    for p in (0.5, 0.8):
        want = None
        for level in (0.0, 0.125, -1.5, 3.0, 11.375, -8.0):
            got, lp, _ = _sample(x + level, f32, temperature=0.9, top_p=p, u=u)
            want = want if want is not None else (got, lp)
            assert np.array_equal(got, want[0]) and np.allclose(lp, want[1], rtol=2.0**-22, atol=0)


@pytest.mark.parametrize("f32", [False, True])
def test_u_of_zero_draws_the_first_token_with_any_mass(f32):
    """The running sum passes 0 with the first kept token whose w is not 0, however small: down to 2^-1000 here."""
    rng = np.random.default_rng([17, f32])
    for n in (60, 3000, 30000):
        x = rng.standard_normal((6, n)) * np.array([1, 3, 20, 50, 100, 2])[:, None]
        x[5] = np.round(x[5] * 2) / 2
        for t in (1.0, 0.3, 0.02):
            x4 = np.maximum(x, x.max(1, keepdims=True) - 650 * t)      # no w in the numbers below 2^-1022
            for par in (dict(top_k=5), dict(top_k=50), dict(top_k=300), dict(top_k=1024), dict(top_k=50, min_p=1e-30), dict(min_p=1e-30),
                        dict(top_k=40, top_p=0.9), dict(top_p=0.999), dict()):
                _check(x4, f32, temperature=t, u=0.0, **par)


@pytest.mark.parametrize("f32", [False, True])
def test_draws_at_exact_ties(f32):
    """A row whose first quarter, half and three quarters hold that share of the mass exactly: u at the share draws the
    token behind it, as the running sum has to exceed u of the whole; u just below it the token before."""
    for n in (4, 8, 24, 48, 96, 240):
        for levels in ((1.5, -2.25), (0.0, 1.0), (7.0, 7.0), (3.0, 2.75)):
            x = np.tile(np.where(np.arange(n // 4) % 2, *levels), 4)[None, :]
            for u, at in ((0.25, n // 4), (0.5, n // 2), (0.75, 3 * n // 4)):
                for par in (dict(top_k=n - 1, min_p=1e-30), dict(min_p=1e-30), dict(top_p=1 - 2.0**-24, min_p=1e-30)):
                    if "top_k" in par:
                        x1 = np.concatenate([x, np.full((1, 1), -np.inf)], 1)
                        par["top_k"] = n
                    else:
                        x1 = x
                    got, _, _ = _sample(x1, f32, temperature=0.7, u=np.float32(u), **par)
                    assert got[0] == at, (n, levels, u, par)
                    got, _, _ = _sample(x1, f32, temperature=0.7, u=np.nextafter(np.float32(u), np.float32(0)), **par)
                    assert got[0] == at - 1, (n, levels, u, par)


@pytest.mark.parametrize("f32", [False, True])
def test_every_row_gets_a_token_where_masses_leave_the_numbers(f32):
    """Parts of a row whose mass is a number while their tokens' alone are not (below 2^-1074 of the largest): masses
    below 2^-1050 may count as none, but a token is drawn."""
    n = 20000
    x = np.full((4, n), -np.inf)
    x[:, :500] = -746.0                      # e^-746 = 2^-1076.3, 500 of them 2^-1067
    x[:, 600] = -740.0
    x[:, n - 1] = 0.0
    x[1, 600:9000] = -np.inf
    x[2, 10000:11000] = -745.0
    x[3, :600] = -np.inf
    for par in (dict(), dict(temperature=1.0, top_p=1.0)):
        got, lp, _ = _sample(x, f32, u=0.0, **par)
        assert got.tolist() == [n - 1] * 4 and (lp == 0).all()


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("temperature", [1.0, 0.1, 0.02, 0.004])
def test_top_k_cuts_among_the_smallest_masses(temperature, f32):
    """A k-th largest logit at 2^-47 of the largest and far below: where k is more than the threads of a work-group, or
    all tokens left are in a few threads' hands.  u = 0 shows a token that ought to be out."""
    rng = np.random.default_rng([int(1000 * temperature), f32])
    x = rng.standard_normal((6, 30000)) * 2
    x[1] = np.round(x[1] * 4) / 4
    x[2, 5000:] = -np.inf                                     # 5000 tokens, in 625 threads' pieces
    x[3, 20000:] = float(_lowest(f32))
    x[4] *= 4
    x[5, 3000:] = -np.inf
    for k in (700, 1025, 2000, 4097, 10000, 25000):
        for u in (0.0, 0.5, 1 - 2.0**-24):
            _check(x, f32, temperature=temperature, top_k=k, u=u)
    _check(x, f32, temperature=temperature, top_k=3000, top_p=0.999, u=0.0)
    _check(x, f32, temperature=temperature, top_k=3000, min_p=1e-30, u=0.0)


@pytest.mark.parametrize("f32", [False, True])
def test_top_p_weighs_the_far_tail(f32):
    """Two equal logits on top and all others 2^-48 or less of them: half of the mass is more than the first alone, if
    only by the tail, and so keeps both."""
    for n in (1000, 30000, 140001):
        for below in (33.5, 34.5, 35.0):
            x = np.full((4, n), 2.0 - below)
            x[:, [n // 7, n // 2]] = 2.0
            _check(x, f32, temperature=1.0, top_p=0.5, u=[0.0, 0.4, 0.6, 0.99])
    low = _lowest(f32)                                        # e^-34 = 2^-49 of the others at this temperature
    x = np.full((4, 30000), low)
    x[:, [100, 20000]] = 5.0
    _check(x, f32, temperature=1e37, top_p=0.5, u=[0.0, 0.4, 0.6, 0.99])


@pytest.mark.parametrize("temperature", [1.0, 0.01, 30.0])
def test_top_p_where_bins_end_between_the_slices(temperature):
    """Rows whose largest logit lies within the reach of single precision's sixteenths (5678 T from 0) and other parts'
    largest just beyond it: those have the same mass to give."""
    rng = np.random.default_rng(18)
    edge = 2.0**17 / (16 * math.log2(math.e)) * temperature
    for n in (20000, 40960, 140001):
        x = rng.standard_normal((6, n)) * temperature
        x = x - x.max(1, keepdims=True) - edge
        x[0, 100] = -edge + 0.01 * temperature               # one token within
        x[1, :5000] += 0.5 * temperature
        x[2, n - 5000:] += 2.0 * temperature
        x[3] += 30 * temperature
        x[4] += 45 * temperature
        for p in (0.3, 0.9, 0.999):
            _check(x, True, temperature=temperature, top_p=p, u=rng.random(6))


@pytest.mark.parametrize("par", [dict(), dict(top_k=1 << 20)])
@pytest.mark.parametrize("depth", [13.9, 14.0, 14.1, 14.3])
def test_top_p_behind_many_tokens_of_little_mass(depth, par):
    """Half a million equal logits between the largest and those the nucleus ends among, in a row too far from 0 for the
    slices' bins, or cut by top_k before: what they weigh together, to less than one of the last."""
    rng = np.random.default_rng([19, int(10 * depth)])
    n, many, last = 524288 + 4000, 524288, 3000
    x = np.full((8, n), -np.inf)
    level = 0.0 if par else -9000.0
    x[:, 0] = level
    x[:, 1:1 + many] = np.float32(level - depth)
    x[:, n - last:] = np.float32(level - depth - 1.5)
    w = np.exp(x[0] - level)
    z, before = w.sum(), w[:1 + many].sum()
    p = np.float32((before + rng.uniform(0.1, 0.9, 8) * (z - before)) / z)
    if par:
        par = dict(top_k=n - 500)                             # the first 2500 of the last ones, and what is -inf never
        x[:, n - last - 600:n - last] = level - depth - 3.0
    _check(x, True, temperature=1.0, top_p=p, u=1 - 2.0**-24, **par)


def test_large_nuclei_draw_the_same_bits_every_time():
    """Nuclei beyond a list: whatever order their last bin's tokens were collected in."""
    rng = np.random.default_rng(20)
    rows, n = 24, 140001
    x = rng.standard_normal((rows, n)) * rng.choice([0.3, 0.8, 1.5], (rows, 1))
    par = dict(temperature=1.0, top_p=rng.uniform(0.6, 0.99, rows), u=rng.random(rows))
    want = _sample(x, True, **par)[:2]
    for _ in range(20):
        got = _sample(x, True, **par)[:2]
        assert all(np.array_equal(a, b) for a, b in zip(got, want))
