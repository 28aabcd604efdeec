"""Attention over the 8-bit cache where scores are large: from those that a float32 sum of several holds no more to the ends of float32."""
import numpy as np
import pytest

from workloads import gen
from test_q8_gpu import _check_decode, _check_prefill, _layer, _run_decode, _run_prefill, _sequence, _slopes

pytestmark = pytest.mark.gpu


def _one_winner(n, order, sign, Hkv, hd, seed):
    """A sequence whose keys lie along dimension 0, any two of them a 2^-7 of the larger and more apart: a softmax of large scores is one position's value."""
    table, codes, expo = _layer([n], Hkv, hd, seed)
    rank = {"up": np.arange(n), "down": np.arange(n)[::-1], "mixed": np.random.RandomState(seed).permutation(n)}[order]
    for p in range(n):
        b, i = table[0, p // 16], p % 16
        codes[b, 0, :, i] = 0
        codes[b, 0, :, i, 0] = sign * (64 + rank[p] % 60)
        expo[b, 0, :, i] = rank[p] // 60
    return table, codes, expo


def _sharp(k, v, q0, p, slope):
    """Softmax of the scores k q0 / sqrt(hd) + slope (j - p) over positions with keys k along dimension 0, in float64, and how far float32 may be off it.

    One weight w of nearly one, which loses its two terms' last bits (2^-22) and has a quotient and three products: 2^-20 of the result.  A score is some
    sixteen roundings of its two parts off, the winner's too, so that another weight is off by the exponential of both.  A weight times its value's unit is
    besides up to half a step of fp16 off, 2^-25, where the largest is held at 2^9 or more."""
    hd = v.shape[1]
    part, bias = np.abs(k * q0) / hd ** 0.5, slope * (np.arange(len(k)) - p)
    s = k * q0 / hd ** 0.5 + bias
    top = s.argmax()
    w = np.exp(s - s[top])
    ref = w @ v / w.sum()
    off = 16 * 2.0 ** -24 * (part + np.abs(bias))
    more = w * np.expm1(np.minimum(off + off[top], 50.0))
    more[top] = 0.0
    most = np.abs(v).max(1)
    unit = np.exp2(np.floor(np.log2(np.where(most > 0, most, 1.0))) - 6)
    step = 2.0 ** -34 * (w * unit).max() * (np.abs(v) / unit[:, None]).sum(0)
    return ref, 2.0 ** -20 * np.abs(ref) + more @ (np.abs(v) + np.abs(ref)) + step


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (64, 4, 1)])
@pytest.mark.parametrize("order,sign", [("up", 1), ("down", 1), ("mixed", 1), ("mixed", -1)])
@pytest.mark.parametrize("size", [12, 20, 25, 33, 60, 75])
@pytest.mark.parametrize("n,before,bias", [(70, 11, False), (70, 11, True), (67, 1903, False), (67, 1903, True)])
def test_prefill_of_large_scores(hd, H, Hkv, order, sign, size, n, before, bias):
    """Scores of 2^size .. 2^(size + 39)."""
    length = before + n
    table, codes, expo = _one_winner(length, order, sign, Hkv, hd, size + n)
    q = np.zeros((n, H, hd), np.float32)
    q[:, :, 0] = 2.0 ** (size - 6) * hd ** 0.5
    slopes = np.minimum(_slopes(H), 2.0 ** (size - 14)) if bias else None
    tiles = [(0, n, before, 0, 0, 0)]
    out = _run_prefill(gen.normal(1, 1, (1,)).new_tensor(q.reshape(n, -1)), n, table, codes, expo, tiles, H, Hkv, hd, length - 1, slopes=slopes)
    got = out.double().cpu().numpy()
    k, v = _sequence(table, codes, expo, 0, length)
    for r in range(0, n, 3):
        end = before + r + 1
        for h in range(H):
            j = h // (H // Hkv)
            ref, bound = _sharp(k[:end, j, 0], v[:end, j], float(q[r, h, 0]), end - 1, float(np.float32(slopes[h])) if bias else 0.0)
            assert (np.abs(got[r, h] - ref) <= bound).all(), (r, h, np.nanmax(np.abs(got[r, h] - ref) / np.maximum(bound, 1e-300)))


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (64, 4, 1)])
@pytest.mark.parametrize("n,before,bias", [(90, 33, False), (65, 1207, False), (65, 1207, True)])
def test_prefill_of_scores_of_any_size(hd, H, Hkv, n, before, bias):
    """Rows whose scores span 2^-4 .. 2^17, side by side."""
    length = before + n
    table, codes, expo = _layer([length], Hkv, hd, n + hd)
    q = gen.normal(n, 13, (n, H * hd)) * (2.0 ** (gen.randint(n, 14, -5, 13, n).double()))[:, None].float()
    tiles = [(0, n, before, 0, 0, 0)]
    kw = dict(slopes=_slopes(H) if bias else None)
    out = _run_prefill(q, n, table, codes, expo, tiles, H, Hkv, hd, length - 1, **kw)
    _check_prefill(out, q, table, codes, expo, tiles, [length], H, Hkv, hd, some=2, **kw)


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (128, 2, 1), (64, 4, 1), (128, 8, 1), (64, 16, 1)])
@pytest.mark.parametrize("order,sign", [("up", 1), ("down", 1), ("mixed", 1), ("mixed", -1)])
@pytest.mark.parametrize("size", [12, 20, 25, 27, 33, 60, 75])
@pytest.mark.parametrize("bias", [False, True])
def test_decode_of_large_scores(hd, H, Hkv, order, sign, size, bias):
    n = 1900
    ctx = [n, n - 1, 700, 64, 63, 17, 2, 1]
    table, codes, expo = _one_winner(n, order, sign, Hkv, hd, size + H)
    q = np.zeros((len(ctx), H, hd), np.float32)
    q[:, :, 0] = 2.0 ** (size - 6) * hd ** 0.5
    slopes = np.minimum(_slopes(H), 2.0 ** (size - 14)) if bias else None
    out = _run_decode(gen.normal(1, 1, (1,)).new_tensor(q.reshape(len(ctx), -1)), table, codes, expo, [0] * len(ctx), ctx, H, Hkv, hd, slopes=slopes)
    got = out.double().cpu().numpy()
    k, v = _sequence(table, codes, expo, 0, n)
    for r, end in enumerate(ctx):
        for h in range(H):
            j = h // (H // Hkv)
            ref, bound = _sharp(k[:end, j, 0], v[:end, j], float(q[r, h, 0]), end - 1, float(np.float32(slopes[h])) if bias else 0.0)
            assert (np.abs(got[r, h] - ref) <= bound).all(), (r, h, np.nanmax(np.abs(got[r, h] - ref) / np.maximum(bound, 1e-300)))


@pytest.mark.parametrize("H,Hkv", [(2, 2), (4, 1)])
@pytest.mark.parametrize("value", [-126, -40, -12, -6, -5, 0, 50])
def test_decode_of_values_of_one_unit_under_large_scores(H, Hkv, value):
    """A score of 7e7 beside smaller ones, under values of each of these units."""
    hd, n = 64, 300
    table, codes, expo = _layer([n], Hkv, hd, 4)
    expo[table[0, :19], 1] = value
    codes[table[0, :19], 0], expo[table[0, :19], 0] = 0, 0
    codes[table[0, 11], 0, :, 3, 0] = 70
    codes[table[0, 4], 0, :, 9, 0] = 69
    q = np.zeros((1, H, hd), np.float32)
    q[:, :, 0] = 8e6
    out = _run_decode(gen.normal(1, 1, (1,)).new_tensor(q.reshape(1, -1)), table, codes, expo, [0], [n], H, Hkv, hd).double().cpu().numpy()
    v = _sequence(table, codes, expo, 0, n)[1][11 * 16 + 3]
    assert (np.abs(out[0] - np.repeat(v, H // Hkv, 0)) <= 2.0 ** -20 * np.abs(np.repeat(v, H // Hkv, 0))).all()


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (64, 4, 1), (128, 16, 1)])
@pytest.mark.parametrize("bias", [False, True])
def test_decode_of_scores_of_any_size(hd, H, Hkv, bias):
    """Rows whose scores span 2^-4 .. 2^17, side by side."""
    ctx = [1300] * 10 + [200] * 9
    table, codes, expo = _layer([1300], Hkv, hd, hd)
    q = gen.normal(hd, 13, (len(ctx), H * hd)) * (2.0 ** (gen.randint(hd, 14, -5, 13, len(ctx)).double()))[:, None].float()
    kw = dict(slopes=_slopes(H) if bias else None)
    out = _run_decode(q, table, codes, expo, [0] * len(ctx), ctx, H, Hkv, hd, **kw)
    _check_decode(out, q, table, codes, expo, [0] * len(ctx), ctx, H, Hkv, hd, **kw)


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (64, 4, 1)])
@pytest.mark.parametrize("size", [3, 20, 26, 33, 60, 100])
@pytest.mark.parametrize("zeros", ["none", "first half", "every other step", "all but a few"])
def test_prefill_of_large_scores_that_are_all_alike(hd, H, Hkv, size, zeros):
    """Equal scores in every share, and values that are zero in some: the mean of the values."""
    n, before = 37, 1830
    length = before + n
    table, codes, expo = _layer([length], Hkv, hd, 31)
    blocks = table[0, :-(-length // 16)]
    codes[blocks, 0], expo[blocks, 0] = 0, 0
    codes[blocks, 0, :, :, 0] = 64
    at = np.arange(length)
    none = {"none": at < 0, "first half": at < 1000, "every other step": at // 64 % 2 == 0, "all but a few": at % 500 != 450}[zeros]
    for p in at[none]:
        codes[table[0, p // 16], 1, :, p % 16], expo[table[0, p // 16], 1, :, p % 16] = 0, -126
    q = np.zeros((n, H, hd), np.float32)
    q[:, :, 0] = 2.0 ** (size - 6) * hd ** 0.5
    out = _run_prefill(gen.normal(1, 1, (1,)).new_tensor(q.reshape(n, -1)), n, table, codes, expo, [(0, n, before, 0, 0, 0)], H, Hkv, hd, length - 1)
    got = out.double().cpu().numpy()
    v = _sequence(table, codes, expo, 0, length)[1]
    for r in range(0, n, 6):
        seen = v[:before + r + 1].repeat(H // Hkv, 1)
        # weights that are the same bits but between shares, whose two largest scores are rounded (2^-24 each where they are not large): sums of 2^11 numbers
        # one after another, 2^-13 at most of the mean magnitude, and as much as one share's weight may be off
        off = 2.0 ** -13 * np.abs(seen).mean(0)
        assert (np.abs(got[r] - seen.mean(0)) <= off).all(), (r, np.abs(got[r] - seen.mean(0)).max())


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (64, 4, 1)])
@pytest.mark.parametrize("small", [-120, -126, -130, -137, -149])
@pytest.mark.parametrize("cap", [0.0, 1e-3])
def test_queries_below_the_normal_numbers(hd, H, Hkv, small, cap):
    """Queries of 2^small, subnormal ones among them, over keys up to 2^120."""
    n, before = 40, 533
    length = before + n
    nb = -(-length // 16)
    table, codes, expo = _layer([length], Hkv, hd, 41)
    expo[table[0, :nb], 0] = np.array([113, 112, 90])[gen.randint(41, 1, 0, 2, nb * Hkv * 16).numpy().reshape(nb, Hkv, 16)]
    q = (gen.normal(41, 13, (n, H * hd)).double() * 2.0 ** small).float()
    assert (q != 0).any()
    tiles = [(0, n, before, 0, 0, 0)]
    out = _run_prefill(q, n, table, codes, expo, tiles, H, Hkv, hd, length - 1, cap=cap)
    _check_prefill(out, q, table, codes, expo, tiles, [length], H, Hkv, hd, some=3, cap=cap)
    rows = [0, 17, 39]
    ctx = [before + r + 1 for r in rows]
    out = _run_decode(q[rows].contiguous(), table, codes, expo, [0] * 3, ctx, H, Hkv, hd, cap=cap)
    _check_decode(out, q[rows].contiguous(), table, codes, expo, [0] * 3, ctx, H, Hkv, hd, cap=cap)
