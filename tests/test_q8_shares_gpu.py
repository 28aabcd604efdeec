"""Prompt attention over the 8-bit cache where a tile's positions are split into shares: chunks behind long sequences, at odd starts, under every mask,
against the plain implementation in 64 bits of test_q8_gpu.py."""
import numpy as np
import pytest

from workloads import gen
from test_q8_gpu import _attend, _check_decode, _check_prefill, _layer, _run_decode, _run_prefill, _sequence, _slopes

pytestmark = pytest.mark.gpu


def _check_rows(out, q, table, codes, expo, tile, length, H, Hkv, hd, rows, window=0):
    """These rows of one sequence's tile against float64; positions of blocks that the table does not map take no part."""
    at, n, pos, s, first, prefix = tile
    mapped = np.array([table[s, p // 16] >= 0 for p in range(length)])
    whole = table.copy()
    whole[s, whole[s] < 0] = 0      # for reading the values: these positions are dropped below
    k, v = _sequence(whole, codes, expo, s, length)
    got = out.double().cpu().numpy()
    for r in rows:
        p = pos + r
        lo, hi = max(first, p - window + 1 if window else 0, 0), min(max(p, prefix - 1), length - 1)
        use = np.arange(lo, hi + 1)[mapped[lo:hi + 1]] if lo <= hi else np.arange(0)
        for h in range(H):
            j = h // (H // Hkv)
            ref, bound = _attend(q[at + r, h * hd:(h + 1) * hd].double().numpy(), k[use, j], v[use, j], 0, 0, len(use) - 1, 0.0, 0.0, least=9)
            g = got[at + r, h]
            assert np.array_equal(np.isnan(g), np.isnan(ref)), (r, h)
            assert (np.abs(g - ref) <= bound)[~np.isnan(ref)].all(), (r, h, np.nanmax(np.abs(g - ref) / np.maximum(bound, 1e-300)))


def _tiles(n, before):
    return [(i, min(128, n - i), before + i, 0, 0, 0) for i in range(0, n, 128)]


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (64, 4, 2)])
@pytest.mark.parametrize("zeros", ["all", "ends of shares", "starts of shares", "all but one"])
@pytest.mark.parametrize("n,before", [(257, 1263), (65, 1999), (128, 500)])
def test_prefill_of_zero_values_over_shares(hd, H, Hkv, zeros, n, before):
    """Values that are zero, as an append stores them (e = -126), over whole 64-position steps: rows whose wave goes on to steps that they do not see."""
    length = before + n
    table, codes, expo = _layer([length], Hkv, hd, n + hd)
    where = np.arange(length)
    none = {"all": where >= 0, "ends of shares": where >= before - 70, "starts of shares": where // 64 % 4 == 0, "all but one": where != 1150 % length}[zeros]
    for p in where[none]:
        codes[table[0, p // 16], 1, :, p % 16], expo[table[0, p // 16], 1, :, p % 16] = 0, -126
    q = gen.normal(n, 13, (n, H * hd))
    tiles = _tiles(n, before)
    out = _run_prefill(q, n, table, codes, expo, tiles, H, Hkv, hd, length - 1)
    assert out.isfinite().all()
    if zeros == "all":
        assert (out == 0).all()
    for t in tiles:
        _check_rows(out, q, table, codes, expo, t, length, H, Hkv, hd, range(0, t[1], 5))


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (64, 4, 2)])
@pytest.mark.parametrize("n,before", [(40, 201), (60, 1900)])
def test_prefill_of_zero_values_before_unmapped_blocks(hd, H, Hkv, n, before):
    """64 zeros, 64 positions that the table does not map, then other values."""
    length = before + n
    table, codes, expo = _layer([length], Hkv, hd, 3 * n)
    for a in (range(0, length, 256) if before > 1000 else (0,)):
        blocks = table[0, a // 16:a // 16 + 4]
        codes[blocks, 1], expo[blocks, 1] = 0, -126
        table[0, a // 16 + 4:a // 16 + 8] = -1
    q = gen.normal(n, 13, (n, H * hd))
    tile = _tiles(n, before)[0]
    out = _run_prefill(q, n, table, codes, expo, [tile], H, Hkv, hd, length - 1)
    _check_rows(out, q, table, codes, expo, tile, length, H, Hkv, hd, range(0, n, 3))


@pytest.mark.parametrize("down", [8.0, 40.0, 60.0])
@pytest.mark.parametrize("n,before", [(40, 201), (60, 1900)])
def test_prefill_of_small_weights_beside_a_zero_value(down, n, before):
    """The position that draws nearly everything has a zero value, the first 64 do: what is left are weights of 2^-down and less."""
    H = Hkv = 2
    hd, length = 128, before + n
    table, codes, expo = _layer([length], Hkv, hd, 5 * n)
    codes[table[0, :4], 1], expo[table[0, :4], 1] = 0, -126
    q = gen.normal(n, 13, (n, H * hd), std=0.02)
    q[:, ::hd] = 8.0
    codes[:, 0, :, :, 0] = 0
    b = table[0, 1]
    codes[b, 0, :, 3], expo[b, 0, :, 3] = 0, 0
    codes[b, 0, :, 3, 0] = round(down * np.log(2.0) * hd ** 0.5 / 8.0)
    tile = _tiles(n, before)[0]
    out = _run_prefill(q, n, table, codes, expo, [tile], H, Hkv, hd, length - 1)
    assert (out != 0).any()
    _check_rows(out, q, table, codes, expo, tile, length, H, Hkv, hd, range(0, n, 3))


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (64, 4, 2)])
@pytest.mark.parametrize("n,before", [(100, 30), (100, 1500)])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, False), (0.0, True)])
def test_prefill_of_queries_that_are_not_finite(hd, H, Hkv, n, before, cap, bias):
    """A head that is not finite gives NaN where its row sees anything, and 0 where it does not: before its document, or in unmapped blocks alone."""
    length = before + n
    table, codes, expo = _layer([length, length], Hkv, hd, n + before)
    table[1, :(before + 60) // 16 + 1] = -1
    q = gen.normal(n, 13, (2 * n, H * hd))
    for r in (0, 5, 31, 40, 90):
        q[r, 3], q[n + r, hd + 1] = float("nan"), float("inf")
    tiles = [(0, n, before, 0, before + 35, 0), (n, n, before, 1, 0, 0)]
    out = _run_prefill(q, 2 * n, table, codes, expo, tiles, H, Hkv, hd, length - 1, cap=cap, slopes=_slopes(H) if bias else None).cpu()
    for r in range(n):
        for head in range(H):
            for s, sees in ((0, r >= 35), (1, before + r > (before + 60) // 16 * 16 + 15)):
                got, nan = out[s * n + r, head], r in (0, 5, 31, 40, 90) and head == s
                assert got.isnan().all() if nan and sees else got.isfinite().all(), (r, head, s)
                assert sees or (got == 0).all(), (r, head, s)


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (64, 4, 1)])
@pytest.mark.parametrize("window,cap,bias", [(0, 0.0, False), (1, 0.0, False), (40, 10.0, False), (0, 30.0, True), (1500, 0.0, True), (900, 5.0, False)])
def test_prefill_segments_over_shares(hd, H, Hkv, window, cap, bias):
    """Chunks behind some 2000 positions that begin and end anywhere, documents that begin in every share, prefixes that reach past the chunk."""
    # (rows, positions before, first visible, prefix) of each sequence
    segs = [(1, 2000, 0, 0), (130, 1987, 0, 0), (33, 2101, 1100, 0), (64, 2037, 2050, 0), (17, 2300, 2310, 0), (100, 1963, 0, 2120), (5, 2015, 2017, 2019),
            (31, 129, 0, 1700), (90, 1791, 700, 1850), (40, 0, 0, 0)]
    lengths = [max(b + n, x) for n, b, _, x in segs]
    table, codes, expo = _layer(lengths, Hkv, hd, hd + H + window)
    tiles, at = [], 1
    for s, (n, before, first, prefix) in enumerate(segs):
        for i in range(0, n, 128):
            tiles.append((at + i, min(128, n - i), before + i, s, first, prefix))
        at += n + s % 3
    q = gen.normal(window + H, 13, (at + 2, H * hd))
    kw = dict(window=window, cap=cap, slopes=_slopes(H) if bias else None)
    out = _run_prefill(q, at + 2, table, codes, expo, tiles, H, Hkv, hd, max(lengths) - 1, **kw)
    _check_prefill(out, q, table, codes, expo, tiles, lengths, H, Hkv, hd, some=5, **kw)
    named = np.zeros(at + 2, bool)
    for t in tiles:
        named[t[0]:t[0] + t[1]] = True
    assert (out.cpu().numpy()[~named] == 9.0).all()


@pytest.mark.parametrize("window", [0, 700])
def test_prefill_keeps_what_is_not_finite_where_it_is_over_shares(window):
    H, Hkv, hd, n, before = 4, 2, 128, 70, 1801
    length = before + n
    table, codes, expo = _layer([length, length], Hkv, hd, 9)
    expo[table[0, 113], 0, 1, 7] = -128      # the key of KV head 1 at position 1815
    expo[table[1, 70], 1, 0, 2] = -128       # the value of KV head 0 at position 1122: in the band of some rows
    q = gen.normal(9, 13, (2 * n, H * hd))
    q[10, 3] = float("nan")
    q[20, 2 * hd + 5] = float("inf")
    tiles = [(s * n, n, before, s, 0, 0) for s in range(2)]
    out = _run_prefill(q, 2 * n, table, codes, expo, tiles, H, Hkv, hd, length - 1, window=window)
    _check_prefill(out, q, table, codes, expo, tiles, [length, length], H, Hkv, hd, window=window, some=2)


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (64, 4, 2)])
def test_prefill_of_unmapped_blocks_over_shares(hd, H, Hkv):
    """Blocks that the table does not map: a whole share's, a step's, single ones, and those at the chunk's own positions."""
    n, before = 100, 1501
    table, codes, expo = _layer([before + n], Hkv, hd, 21)
    table[0, [*range(16, 33), *range(40, 44), 50, 61, 62, 95]] = -1
    q = gen.normal(21, 13, (n, H * hd))
    tile = (0, n, before, 0, 0, 0)
    out = _run_prefill(q, n, table, codes, expo, [tile], H, Hkv, hd, before + n - 1)
    _check_rows(out, q, table, codes, expo, tile, before + n, H, Hkv, hd, range(0, n, 4))


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (64, 4, 1)])
@pytest.mark.parametrize("zeros", [False, True])
def test_keys_and_values_near_the_ends_of_their_range_over_shares(hd, H, Hkv, zeros):
    """Keys up to 2^120 under queries of 2^-115, and keys of 2^-120 and 2^-104 under queries of 2^108; values over 2^84, zeros first in every share."""
    n, before = 70, 1777
    length = before + n
    nb = -(-length // 16)
    for keys, small in (((113, 100, 90), -115), ((-126, -124, -110), 108)):
        table, codes, expo = _layer([length], Hkv, hd, 18)
        pick = gen.randint(18, 1, 0, len(keys) - 1, nb * Hkv * 16).numpy().reshape(nb, Hkv, 16)
        expo[table[0, :nb], 0] = np.array(keys)[pick]
        expo[table[0, :nb], 1] = gen.randint(18, 2, -42, 42, nb * Hkv * 16).numpy().reshape(nb, Hkv, 16)
        if zeros:
            for a in range(0, nb, 16):
                codes[table[0, a:a + 4], 1] = 0
                expo[table[0, a:a + 4], 1] = -126
        q = (gen.normal(18, 13, (n, H * hd)).double() * 2.0 ** small).float()
        tiles = [(0, n, before, 0, 0, 0)]
        out = _run_prefill(q, n, table, codes, expo, tiles, H, Hkv, hd, length - 1)
        _check_prefill(out, q, table, codes, expo, tiles, [length], H, Hkv, hd, some=3)


@pytest.mark.parametrize("H,Hkv", [(2, 2), (4, 1), (16, 1)])
@pytest.mark.parametrize("unit", [121, 100, -110, -126])
@pytest.mark.parametrize("size", [1.0, 1e-3])
def test_values_at_the_ends_of_float32(H, Hkv, unit, size):
    """Values of one unit, up to the largest that float32 holds, whose weights are many and alike: every sum stays within the values."""
    hd, n, before = 64, 40, 1777
    length = before + n
    table, codes, expo = _layer([length], Hkv, hd, 22)
    expo[table[0, :-(-length // 16)], 1] = unit
    q = gen.normal(22, 13, (n, H * hd), std=size)
    tiles = [(0, n, before, 0, 0, 0)]
    out = _run_prefill(q, n, table, codes, expo, tiles, H, Hkv, hd, length - 1)
    _check_prefill(out, q, table, codes, expo, tiles, [length], H, Hkv, hd, some=5)
    rows = [0, 3, 39]
    ctx = [before + r + 1 for r in rows]
    out = _run_decode(q[rows].contiguous(), table, codes, expo, [0] * 3, ctx, H, Hkv, hd)
    _check_decode(out, q[rows].contiguous(), table, codes, expo, [0] * 3, ctx, H, Hkv, hd)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("before", [0, 1920])
@pytest.mark.parametrize("down", [26.4, 29.3, 31.2, 33.7])
def test_prefill_of_small_weights_beside_a_small_unit(hd, before, down):
    """One position draws all but 2^-down, its value has a quarter of the others' unit and zeros where theirs count: their weights lose 2^-38 of the largest
    product at most."""
    H, Hkv, n = 2, 1, 12
    length = before + n
    table, codes, expo = _layer([length], Hkv, hd, int(down))
    b = table[0, before // 16]
    codes[b, 0], expo[b, 0] = 0, 0
    codes[b, 0, :, 0, 0], expo[b, 0, :, 0] = 127, 0
    codes[b, 1, :, 0], expo[b, 1] = 0, -6
    codes[b, 1, :, 0, 0], expo[b, 1, :, 0] = 127, -8
    q = gen.normal(int(down), 13, (n, H * hd), std=0.01)
    q[:, ::hd] = float(down * np.log(2.0) * hd ** 0.5 / 127)
    out = _run_prefill(q, n, table, codes, expo, [(0, n, before, 0, before, 0)], H, Hkv, hd, length - 1)
    k, v = _sequence(table, codes, expo, 0, length)
    for r in range(n):
        for h in range(H):
            ref, bound = _attend(q[r, h * hd:(h + 1) * hd].double().numpy(), k[before:before + r + 1, 0], v[before:before + r + 1, 0], 0, 0, r, 0.0, 0.0, least=13)
            assert (np.abs(out[r, h].double().cpu().numpy() - ref) <= bound).all(), (r, h, (np.abs(out[r, h].double().cpu().numpy() - ref) / bound).max())


@pytest.mark.parametrize("hd,H,Hkv", [(128, 4, 2), (64, 8, 2)])
@pytest.mark.parametrize("n,before", [(60, 64), (100, 65), (90, 1600)])
def test_prefill_behind_zero_values_is_as_exact(hd, H, Hkv, n, before):
    """Zero values in the first 64 positions of a share; queries so small that the bound is that of the weights' own roundings."""
    length = before + n
    table, codes, expo = _layer([length], Hkv, hd, n)
    for p in range(length):
        if p // 64 % 4 == 0 or before > 1000 and p < before:
            codes[table[0, p // 16], 1, :, p % 16], expo[table[0, p // 16], 1, :, p % 16] = 0, -126
    q = gen.normal(n, 13, (n, H * hd), std=0.02)
    tile = _tiles(n, before)[0]
    out = _run_prefill(q, n, table, codes, expo, [tile], H, Hkv, hd, length - 1)
    _check_rows(out, q, table, codes, expo, tile, length, H, Hkv, hd, range(n))
