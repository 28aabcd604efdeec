"""The 8-bit cache (append with head norms and rotation, moves) and the attention that reads it on the GPU, against plain implementations in 64 bits
written here."""
import math

import numpy as np
import pytest
import torch

import paper_2406_00059_amd as ld
from workloads import gen
from helpers import device_pool, logical_pool

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(v):
    return torch.as_tensor(np.ascontiguousarray(v), dtype=torch.int32, device=DEV)


def _q8(x):
    """Codes and exponents of float64 vectors [.., hd]; -128 for one that is not finite."""
    x = np.asarray(x, np.float64)
    with np.errstate(all="ignore"):
        top = np.abs(x).max(-1)
        fine = np.isfinite(top) & (top < 2.0 ** 128)
        e = np.where(top > 0, np.floor(np.log2(np.where(fine & (top > 0), top, 1.0))), -1000)
        # log2 next to a power of two may round up to it
        e = np.where(fine & (top > 0) & (np.exp2(np.maximum(e, -1000)) > top), e - 1, e)
        e = np.where(fine, np.maximum(e - 6, -126), -128).astype(np.int64)
        c = np.clip(np.rint(np.where(fine[..., None], x, 0.0) * np.exp2(-e.astype(np.float64))[..., None]), -127, 127)
    return np.where(fine[..., None], c, 0).astype(np.int8), e.astype(np.int8)


def _values(codes, expo):
    e = expo.astype(np.float64)
    return np.where(expo[..., None] == -128, np.nan, codes.astype(np.float64) * np.exp2(np.where(expo == -128, 0.0, e))[..., None])


def _device_layer(codes, expo):
    """Logical codes [n, 2, Hkv, 16, hd] and exponents to the layer's memory image on the device."""
    return device_pool(torch.as_tensor(codes)).contiguous().to(DEV), torch.as_tensor(expo).to(DEV)


def _logical(codes, expo):
    return logical_pool(codes.cpu()).numpy(), expo.cpu().numpy()


def _tables(lengths, seed, spare=0, width=None):
    """Block table of sequences of these lengths in a seeded order of a pool with `spare` blocks of nobody; the pool's blocks."""
    nb = [-(-n // 16) for n in lengths]
    total = sum(nb) + spare
    perm = np.random.RandomState(seed).permutation(total)
    table = np.full((len(lengths), width or max(max(nb), 1)), -1, np.int32)
    at = 0
    for s, n in enumerate(nb):
        table[s, :n] = perm[at:at + n]
        at += n
    return table, total


def _close(got, ref, bound):
    got = got.detach().double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    ok = ~np.isnan(ref)
    off = np.abs(got[ok] - ref[ok])
    assert (off <= bound[ok]).all(), f"{(off / np.maximum(bound[ok], 1e-300)).max()} times the bound"


# ---------------------------------------------------------------- angles

@pytest.mark.parametrize("rot,scaling", [(2, {}), (64, {}), (128, {}), (22, {}), (128, dict(factor=8.0)), (64, dict(factor=4.0, attention=1.25)),
                                         (128, dict(factor=8.0, low=1.0, high=4.0, original=8192)),
                                         (96, dict(factor=32.0, low=0.5, high=0.75, original=77, attention=0.5))])
def test_scaled_angles(rot, scaling):
    pos = np.array([0, 1, 2, 15, 16, 1000, 4095, 131071, 1 << 20, (1 << 31) - 1, 77])
    out = torch.full((len(pos), rot // 2, 2), 5.0, device=DEV)
    ld.ldk_rope_table_scaled(_i32(pos), rot, 10000.0, out, **scaling)
    f = 10000.0 ** (-2.0 * np.arange(rot // 2) / rot)
    g = np.zeros_like(f)
    if scaling.get("original"):
        g = np.clip((scaling["original"] * f / (2 * math.pi) - scaling["low"]) / (scaling["high"] - scaling["low"]), 0, 1)
    f = f * ((1 - g) / scaling.get("factor", 1.0) + g)
    angle = pos[:, None] * f
    size = scaling.get("attention", 1.0)
    ref = size * np.stack([np.cos(angle), np.sin(angle)], -1)
    # one rounding to float32, and an angle whose frequency is some 2^-52 times (1 + 13.3 ln 2) off on either side
    _close(out, ref, 2.0 ** -24 * np.abs(ref) + size * (64 * 2.0 ** -52 * np.abs(angle)[..., None] + 1e-15))


@pytest.mark.parametrize("hd", [64, 128])
def test_angles_without_scaling_are_those_of_the_plain_table(hd):
    pos = _i32([0, 1, 17, 4097, 131071])
    a, b = torch.empty((5, hd // 2, 2), device=DEV), torch.empty((5, hd // 2, 2), device=DEV)
    ld.ldk_rope_table(pos, hd, 10000.0, a)
    ld.ldk_rope_table_scaled(pos, hd, 10000.0, b)
    assert (a.double() - b.double()).abs().max().item() <= 2.0 ** -23      # each rounded once


# ---------------------------------------------------------------- append

def _append_reference(qkv, pos, slot, table, cos_sin, H, Hkv, hd, rot, interleaved, q_gain, k_gain, eps, codes, expo):
    """q in float64; codes and expo (logical) are brought up to date."""
    T = len(pos)
    x = qkv.double().numpy().reshape(T, H + 2 * Hkv, hd).copy()
    with np.errstate(all="ignore"):
        for heads, gain in ((slice(0, H), q_gain), (slice(H, H + Hkv), k_gain)):
            if gain is not None:
                h = x[:, heads]
                x[:, heads] = h / np.sqrt((h ** 2).mean(-1, keepdims=True) + float(np.float32(eps))) * gain.double().numpy()
        i = np.arange(rot // 2)
        one, two = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        if rot:
            cs = cos_sin.double().numpy().reshape(T, rot // 2, 2)
            a, b = x[:, :H + Hkv, one], x[:, :H + Hkv, two]
            c, s = cs[:, None, :, 0], cs[:, None, :, 1]
            x[:, :H + Hkv, one], x[:, :H + Hkv, two] = a * c - b * s, a * s + b * c
    for t, p in enumerate(pos):
        b = table[slot[t], p // 16] if p >= 0 and p // 16 < table.shape[1] else -1
        if b < 0:
            continue
        for kind, heads in ((0, slice(H, H + Hkv)), (1, slice(H + Hkv, None))):
            codes[b, kind, :, p % 16], expo[b, kind, :, p % 16] = _q8(x[t, heads])
    return x[:, :H].reshape(T, H * hd)


def _rows(kind, seed):
    """Positions and sequences of a call's rows."""
    if kind == "one":
        return [37], [0]
    if kind == "batch":      # one row of each of several sequences, among them the first position of a block and the last
        return [0, 15, 16, 31, 63, 5, 100], list(range(7))
    if kind == "chunk":      # a chunk that begins and ends inside blocks
        return list(range(21, 21 + 45)), [0] * 45
    pos = list(range(3, 40)) + [200, 16] + list(range(0, 33)) + [-1, 77, -5]      # chunks, single rows, padding
    return pos, [0] * 37 + [1, 2] + [3] * 33 + [0, 4, 9]


@pytest.mark.parametrize("hd,H,Hkv", [(64, 4, 4), (128, 4, 4), (128, 8, 2), (64, 5, 1), (128, 40, 40)])
@pytest.mark.parametrize("kind", ["one", "batch", "chunk", "mixed"])
@pytest.mark.parametrize("rot,interleaved,norm", [("all", False, ""), ("all", True, "qk"), ("half", False, "qk"), ("odd", True, ""), ("odd", False, "k"), ("none", False, "q")])
def test_append(hd, H, Hkv, kind, rot, interleaved, norm):
    rot = {"all": hd, "half": hd // 2, "odd": 22, "none": 0}[rot]
    seed = hd + H + rot
    pos, slot = _rows(kind, seed)
    T = len(pos)
    table, total = _tables([240] * 10, seed)
    table[4, 77 // 16] = -1      # a block that is not mapped: nothing is written
    qkv = gen.normal(seed, 1, (T, (H + 2 * Hkv) * hd))
    qkv[:, 3::64] *= 6.0
    cos_sin = gen.normal(seed, 2, (T, rot // 2, 2)) if rot else None      # any numbers will do
    gains = [gen.normal(seed, 3 + i, (hd,), std=0.1, mean=1.0) if c in norm else None for i, c in enumerate("qk")]
    codes, expo = np.full((total, 2, Hkv, 16, hd), 77, np.int8), np.full((total, 2, Hkv, 16), 55, np.int8)
    dc, de = _device_layer(codes, expo)
    q = torch.full((T, H * hd), 7.0, device=DEV)
    dev = lambda t: None if t is None else t.to(DEV)      # noqa: E731
    args = (dev(cos_sin), _i32(pos), _i32(slot), _i32(table), dc, de, H, Hkv, hd)
    more = dict(rot=rot, interleaved=interleaved, q_gain=dev(gains[0]), k_gain=dev(gains[1]), eps=1e-5)
    ld.ldk_rope_kv_write_q8(qkv.to(DEV), *args, q, **more)
    ref = _append_reference(qkv, pos, slot, table, cos_sin, H, Hkv, hd, rot, interleaved, *gains, 1e-5, codes, expo)
    got_c, got_e = _logical(dc, de)
    assert np.array_equal(got_e, expo) and np.array_equal(got_c, codes)
    pad = np.array(pos) < 0
    got = q.cpu()
    assert (got[pad] == 7.0).all()
    # half a step of float32; float64's own roundings are 2^-29 of that, of the pair's larger element
    size = np.abs(ref).max(-1, keepdims=True)
    assert (np.abs(got.double().numpy() - ref) <= 2.0 ** -24 * np.abs(ref) + 2.0 ** -48 * size)[~pad].all()
    # in place, and with rows that are further apart
    wide = torch.full((T, (H + 2 * Hkv) * hd + 36), 3.0, device=DEV)
    wide[:, :qkv.shape[1]] = qkv.to(DEV)
    before = wide.clone()
    dc.fill_(77)
    ld.ldk_rope_kv_write_q8(wide, *args, wide, **more)
    assert torch.equal(wide[~torch.as_tensor(pad)][:, :H * hd].cpu(), got[~torch.as_tensor(pad)])
    assert torch.equal(wide[:, H * hd:], before[:, H * hd:]) and torch.equal(wide[torch.as_tensor(pad)], before[torch.as_tensor(pad)])
    assert np.array_equal(_logical(dc, de)[0], got_c)


def test_append_of_vectors_of_any_magnitude():
    """Zero, subnormal, huge, next to powers of two, ties, NaN and infinities: keys without rotation and values."""
    hd = 64
    x = torch.zeros((16, hd))
    x[1] = torch.linspace(-3e-42, 3e-42, hd)
    x[2] = torch.linspace(-3e38, 3e38, hd)
    x[3, 5] = 64.0
    x[4] = torch.arange(hd) + 0.5                    # unit 2^-1 (63.5 of 32 .. 64): no tie; twice that below
    x[5] = torch.arange(hd) * 2 + 0.5                # unit 1: ties to even, 126.5 stays in range
    x[6, :3] = torch.tensor([127.75, -127.75, 127.5])      # rounds past 127: held there
    x[7, 9] = float("nan")
    x[8, 60] = float("inf")
    x[9, 0] = -float("inf")
    x[10, 1] = float(np.nextafter(np.float32(64), np.float32(0)))
    x[11, 1] = 2.0 ** -126
    x[12, 63] = 1e-45
    x[13] = -127.0
    x[14, 7] = float(np.finfo(np.float32).max)
    x[15] = gen.normal(1, 1, (hd,)) * 1e-39
    qkv = torch.cat([torch.zeros(16, hd), x, x.flip(0)], 1).contiguous()
    codes, expo = np.zeros((1, 2, 1, 16, hd), np.int8), np.zeros((1, 2, 1, 16), np.int8)
    dc, de = _device_layer(codes, expo)
    q = torch.empty((16, hd), device=DEV)
    table = np.zeros((1, 1), np.int32)
    ld.ldk_rope_kv_write_q8(qkv.to(DEV), None, _i32(np.arange(16)), _i32([0] * 16), _i32(table), dc, de, 1, 1, hd, q, rot=0)
    codes[0, 0, 0], expo[0, 0, 0] = _q8(x.double().numpy())
    codes[0, 1, 0], expo[0, 1, 0] = _q8(x.double().numpy()[::-1])
    got_c, got_e = _logical(dc, de)
    assert np.array_equal(got_e, expo) and np.array_equal(got_c, codes)
    assert got_e[0, 0, 0, 7] == got_e[0, 0, 0, 8] == got_e[0, 0, 0, 9] == -128 and got_c[0, 0, 0, 5, 0] == 0 and got_c[0, 0, 0, 5, 1] == 2


def test_append_of_queries_that_are_not_finite():
    hd, H = 128, 2
    qkv = gen.normal(3, 1, (2, 4 * hd))
    qkv[0, 5], qkv[1, hd + 7] = float("nan"), float("inf")
    dc, de = _device_layer(np.zeros((1, 2, 1, 16, hd), np.int8), np.zeros((1, 2, 1, 16), np.int8))
    q = torch.zeros((2, H * hd), device=DEV)
    cs = torch.ones((2, hd // 2, 2), device=DEV)
    ld.ldk_rope_kv_write_q8(qkv.to(DEV), cs, _i32([0, 1]), _i32([0, 0]), _i32([[0]]), dc, de, H, 1, hd, q, q_gain=torch.ones(hd, device=DEV), eps=1e-5)
    assert q[0, :hd].isnan().all() and q[0, hd:].isfinite().all() and q[1, :hd].isfinite().all() and q[1, hd:].isnan().any()


# ---------------------------------------------------------------- moves

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hd,Hkv", [(64, 4), (128, 1), (128, 5)])
@pytest.mark.parametrize("ranges", [[(0, 0, 1)], [(1, 5, 6)], [(0, 0, 100), (1, 17, 80), (2, 16, 32)], [(2, 3, 14), (0, 15, 17), (1, 0, 96)]])
def test_moves_there_and_back(dtype, hd, Hkv, ranges):
    lengths = [100, 96, 33]
    table, total = _tables(lengths, 1, spare=2)
    table8, total8 = _tables(lengths, 2, spare=5, width=9)
    logical = gen.normal(hd + Hkv, 1, (total, 2, Hkv, 16, hd)) * torch.exp2(gen.randint(4, 1, -20, 20, total * 2 * Hkv * 16).view(total, 2, Hkv, 16, 1).float())
    logical = logical.to(dtype)
    logical[table[0, 0], 0, 0, 0, 3] = float("nan")
    codes, expo = np.full((total8, 2, Hkv, 16, hd), 9, np.int8), np.full((total8, 2, Hkv, 16), 11, np.int8)
    dc, de = _device_layer(codes, expo)
    pool = device_pool(logical).contiguous().to(DEV)
    most = max(e - f for _, f, e in ranges)
    ld.ldk_kv_to_q8(pool, _i32(table), dc, de, _i32(table8), _i32(ranges), most, Hkv, hd)
    back = torch.full_like(pool, 3.0)
    ref = torch.full_like(logical, 3.0)
    for s, f, e in ranges:
        for p in range(f, e):
            b, b8 = table[s, p // 16], table8[s, p // 16]
            codes[b8, :, :, p % 16], expo[b8, :, :, p % 16] = _q8(logical[b, :, :, p % 16].double().numpy())
            ref[b, :, :, p % 16] = torch.as_tensor(_values(codes[b8, :, :, p % 16], expo[b8, :, :, p % 16])).to(dtype)
    got_c, got_e = _logical(dc, de)
    assert np.array_equal(got_e, expo) and np.array_equal(got_c, codes)
    ld.ldk_kv_from_q8(dc, de, _i32(table8), back, _i32(table), _i32(ranges), most, Hkv, hd)
    got = logical_pool(back.cpu())
    assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.nan_to_num(0.0), ref.nan_to_num(0.0))      # exact in both types
    # what went through the pool keeps its codes
    again, again_e = dc.clone(), de.clone()
    ld.ldk_kv_to_q8(back, _i32(table), again, again_e, _i32(table8), _i32(ranges), most, Hkv, hd)
    assert torch.equal(again, dc) and torch.equal(again_e, de)


def test_moves_leave_out_unmapped_blocks_and_positions_past_max_len():
    hd, Hkv = 128, 2
    table, table8 = np.array([[0, 1, -1, 3]], np.int32), np.array([[0, -1, 2, 3]], np.int32)
    logical = gen.normal(1, 1, (4, 2, Hkv, 16, hd))
    codes, expo = np.full((4, 2, Hkv, 16, hd), 9, np.int8), np.full((4, 2, Hkv, 16), 11, np.int8)
    dc, de = _device_layer(codes, expo)
    ld.ldk_kv_to_q8(device_pool(logical).contiguous().to(DEV), _i32(table), dc, de, _i32(table8), _i32([[0, 2, 500]]), 52, Hkv, hd)
    for p in (*range(2, 16), *range(48, 54)):      # 2 .. 53, without the blocks that one side does not map
        codes[p // 16, :, :, p % 16], expo[p // 16, :, :, p % 16] = _q8(logical[p // 16, :, :, p % 16].double().numpy())
    got_c, got_e = _logical(dc, de)
    assert np.array_equal(got_e, expo) and np.array_equal(got_c, codes)


# ---------------------------------------------------------------- attention

U = 2.0 ** -24      # half a step of float32 at 1


def _attend(q, k, v, p, lo, hi, cap, slope, least=13):
    """One row and head in float64 over positions lo .. hi of k, v [positions, hd]; the result, and how far float32 may be off it.

    A score is at most 2^-23 of max |q| sum |k| / sqrt(hd) off by the query's 24 bits under its largest element, some eight roundings of that size by
    its sums, scales and conversions, eight of the capped score, four of the bias; a weight some sixteen roundings (the exponential's argument and its
    result, its two 11-bit halves, the value's unit) and as many as its distance from the top in the argument; the sum one each 64 positions.
    The halves are fp16 numbers whose smallest step is 2^-24, and the largest p 2^e is held at 2^least or more (the decode kernel: 2^13, the one for prompt
    rows, which scales less often: 2^9): a weight times its value's unit is besides up to half a step off, 2^-25 2^-least max p 2^e.  That shows where the value that draws everything has a
    code of zero (a weight of 4e-10 was 0.8 % off beside one of 1)."""
    hd = len(q)
    lo, hi = max(lo, 0), min(hi, len(k) - 1)
    if hi < lo:
        return np.zeros(hd), np.zeros(hd)
    if not np.isfinite(q).all():
        return np.full(hd, np.nan), np.zeros(hd)
    k, v = k[lo:hi + 1], v[lo:hi + 1]
    if np.isnan(k).any() or np.isnan(v).any():
        return np.full(hd, np.nan), np.zeros(hd)
    s = k @ q / math.sqrt(hd)
    off = 10 * np.abs(q).max() * np.abs(k).sum(1) / math.sqrt(hd)
    if cap:
        s = cap * np.tanh(s / cap)
        off = off + 8 * np.abs(s)
    bias = slope * (np.arange(lo, hi + 1) - p)
    s = s + bias
    off = off + 4 * np.abs(bias)
    w = np.exp(s - s.max())
    w /= w.sum()
    off = U * (off + 16 + 2 * np.abs(s - s.max()) + 8 + len(s) / 64)
    off = np.minimum(off, 1e3)
    out = w @ v
    top = np.abs(v).max(1)
    unit = np.exp2(np.where(top > 0, np.floor(np.log2(np.where(top > 0, top, 1.0))) - 6, -126.0))
    step = 2.0 ** (-25 - least) * (w * unit).max() * (np.abs(v) / unit[:, None]).sum(0)
    return out, (w * off) @ np.abs(v) + np.abs(out) * (w @ off) + step + 1e-30


def _layer(lengths, Hkv, hd, seed, spare=3, width=None):
    """Table, codes and exponents of random sequences: keys with a few large dimensions; unwritten slots hold NaN marks and wild codes."""
    table, total = _tables(lengths, seed, spare, width)
    x = gen.normal(seed, 11, (total, 2, Hkv, 16, hd)).double().numpy()
    x[:, 0, :, :, 5::32] *= 4.0
    codes, expo = _q8(x * np.exp2(gen.randint(seed, 12, -3, 2, total * 2 * Hkv * 16).numpy().reshape(total, 2, Hkv, 16, 1).astype(np.float64)))
    owned = np.zeros((total, 16), bool)
    for s, n in enumerate(lengths):
        for b in range(-(-n // 16)):
            owned[table[s, b], :min(16, n - 16 * b)] = True
    codes = np.where(owned[:, None, None, :, None], codes, np.int8(-128))
    expo = np.where(owned[:, None, None], expo, np.int8(-128))
    return table, codes, expo


def _sequence(table, codes, expo, s, n):
    """Keys and values [n, Hkv, hd] of a sequence."""
    blocks = table[s, :-(-n // 16)]
    x = _values(codes[blocks], expo[blocks])      # [nb, 2, Hkv, 16, hd]
    x = x.transpose(1, 0, 3, 2, 4).reshape(2, -1, x.shape[2], x.shape[4])
    return x[0, :n], x[1, :n]


def _slopes(H):
    return 2.0 ** (-8.0 * (np.arange(H) + 1) / H)


def _f32(v):
    return torch.as_tensor(v, dtype=torch.float32, device=DEV)


def _run_decode(q, table, codes, expo, slot, ctx, H, Hkv, hd, window=0, first=None, cap=0.0, slopes=None, max_ctx=None, spare=0, q_stride=None):
    dc, de = _device_layer(codes, expo)
    T = len(ctx)
    max_ctx = max(ctx) if max_ctx is None else max_ctx
    out = torch.full((T, H, hd), 9.0, device=DEV)
    n = ld.ldk_attention_q8_scratch_bytes(T, H, Hkv, hd, max_ctx, window)
    scratch = torch.full((n + spare,), 255, dtype=torch.uint8, device=DEV)      # NaN patterns: nothing in it has to be clear
    ld.ldk_paged_attention_q8(q.to(DEV), q_stride or H * hd, dc, de, _i32(table), _i32(slot), _i32(ctx), max_ctx, H, Hkv, hd, out, scratch, window=window,
                              first=None if first is None else _i32(first), softcap=cap, slopes=None if slopes is None else _f32(slopes))
    return out


def _check_decode(out, q, table, codes, expo, slot, ctx, H, Hkv, hd, window=0, first=None, cap=0.0, slopes=None):
    ref, bound = np.zeros((len(ctx), H, hd)), np.zeros((len(ctx), H, hd))
    qd = q.double().numpy().reshape(len(ctx), -1)
    for t, n in enumerate(ctx):
        if n == 0:
            continue
        k, v = _sequence(table, codes, expo, slot[t], n)
        lo = max(first[t] if first is not None else 0, n - window if window else 0)
        for h in range(H):
            j = h // (H // Hkv)
            ref[t, h], bound[t, h] = _attend(qd[t, h * hd:(h + 1) * hd], k[:, j], v[:, j], n - 1, lo, n - 1, cap,
                                             float(np.float32(slopes[h])) if slopes is not None else 0.0)
    _close(out, ref, bound)
    return ref


LENGTHS = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 257, 700]


@pytest.mark.parametrize("hd,H,Hkv", [(64, 4, 4), (128, 4, 4), (128, 8, 2), (64, 6, 2), (128, 8, 1), (128, 5, 1), (64, 16, 1), (128, 34, 2), (64, 33, 1)])
@pytest.mark.parametrize("window,cap,bias,doc", [(0, 0.0, False, False), (1, 0.0, False, False), (50, 20.0, False, True), (0, 5.0, True, False), (129, 0.0, True, True)])
def test_decode(hd, H, Hkv, window, cap, bias, doc):
    table, codes, expo = _layer(LENGTHS, Hkv, hd, hd + H)
    T = len(LENGTHS)
    q = gen.normal(H, 13, (T, H * hd)) * torch.exp2(gen.randint(H, 14, -2, 2, T).float())[:, None]
    first = [n // 2 if t % 3 else (n if t % 2 else n + 40) for t, n in enumerate(LENGTHS)] if doc else None      # also rows that see nothing
    kw = dict(window=window, first=first, cap=cap, slopes=_slopes(H) if bias else None)
    out = _run_decode(q, table, codes, expo, range(T), LENGTHS, H, Hkv, hd, **kw)
    _check_decode(out, q, table, codes, expo, range(T), LENGTHS, H, Hkv, hd, **kw)


@pytest.mark.parametrize("T,H,Hkv,hd", [(1, 4, 1, 128), (2, 2, 2, 128), (1, 32, 8, 128), (3, 4, 4, 64)])
@pytest.mark.parametrize("n", [1500, 4097, 20011])
def test_decode_of_few_rows_over_long_sequences(T, H, Hkv, hd, n):
    lengths = [n - 37 * t for t in range(T)]
    table, codes, expo = _layer(lengths, Hkv, hd, n)
    q = gen.normal(n, 13, (T, H * hd))
    out = _run_decode(q, table, codes, expo, range(T), lengths, H, Hkv, hd, spare=1000)
    _check_decode(out, q, table, codes, expo, range(T), lengths, H, Hkv, hd)
    # a band whose first block is far inside, and the blocks below it given up
    w = 1000
    cut = table.copy()
    for t, m in enumerate(lengths):
        cut[t, :(m - w) // 16] = -1
    banded = _run_decode(q, cut, codes, expo, range(T), lengths, H, Hkv, hd, window=w)
    _check_decode(banded, q, table, codes, expo, range(T), lengths, H, Hkv, hd, window=w)


def test_decode_shares_sequences_and_takes_strided_queries():
    """Several rows of one sequence at different lengths, out of order; queries inside wider rows at an odd address."""
    H, Hkv, hd = 8, 2, 128
    table, codes, expo = _layer([300, 40], Hkv, hd, 5, width=30)
    slot, ctx = [0, 1, 0, 0, 1], [300, 40, 1, 299, 7]
    stride = H * hd + 5
    q = gen.normal(5, 13, (5 * stride,))
    wide = torch.zeros(5 * stride + 1, device=DEV)[1:]
    wide.copy_(q)
    out = _run_decode(wide, table, codes, expo, slot, ctx, H, Hkv, hd, q_stride=stride, max_ctx=400)
    _check_decode(out, q.view(5, stride)[:, :H * hd].contiguous(), table, codes, expo, slot, ctx, H, Hkv, hd)


def test_decode_of_weights_and_units_of_any_size():
    """One position far above the others, values of units 2^-40 and 2^40 side by side, huge and tiny queries, keys all zero."""
    H = Hkv = 2
    hd, n = 128, 333
    table, codes, expo = _layer([n] * 6, Hkv, hd, 6)
    for s in range(6):
        b = table[s, 9]
        if s == 0:
            codes[b, 0, :, 3] = 127      # a key that draws everything
        if s == 1:
            expo[table[s, :20], 1] = gen.randint(6, 1, -40, 30, 20 * Hkv * 16).numpy().reshape(20, Hkv, 16)
        if s == 2:
            codes[table[s], 0] = 0
            expo[table[s], 0] = np.where(expo[table[s], 0] == -128, -128, -126)
        if s == 5:
            expo[table[s, :20], 1] = -126
    q = gen.normal(6, 13, (6, H * hd)).abs() * torch.tensor([3.0, 1.0, 1.0, 1e-30, 40.0, 1.0])[:, None]
    q[3, 5] = 0.0
    out = _run_decode(q, table, codes, expo, range(6), [n] * 6, H, Hkv, hd)
    _check_decode(out, q, table, codes, expo, range(6), [n] * 6, H, Hkv, hd)
    zero = _run_decode(q * 0, table, codes, expo, range(6), [n] * 6, H, Hkv, hd)
    _check_decode(zero, q * 0, table, codes, expo, range(6), [n] * 6, H, Hkv, hd)


def test_decode_keeps_what_is_not_finite_where_it_is():
    H, Hkv, hd = 4, 2, 64
    lengths = [200, 200, 200, 200]
    table, codes, expo = _layer(lengths, Hkv, hd, 7)
    expo[table[1, 3], 0, 1, 5] = -128      # a key of KV head 1 at position 53
    expo[table[2, 0], 1, 0, 0] = -128      # a value of KV head 0 at position 0
    q = gen.normal(7, 13, (4, H * hd))
    q[0, 5], q[3, hd + 1], q[3, 3 * hd] = float("nan"), float("inf"), -float("inf")
    for first in (None, [0, 54, 1, 0], [0, 53, 0, 200]):
        out = _run_decode(q, table, codes, expo, range(4), lengths, H, Hkv, hd, first=first)
        ref = _check_decode(out, q, table, codes, expo, range(4), lengths, H, Hkv, hd, first=first)
        assert np.isnan(ref).any() and np.isfinite(ref).any()


def test_decode_of_blocks_past_two_and_four_gigabytes():
    """Blocks whose bytes begin past 2^31 and 2^32."""
    H = Hkv = 32
    hd, n = 128, 40
    each = 2 * Hkv * 16 * hd
    total = (1 << 32) // each + 5
    codes = torch.empty((total, 2, Hkv, 16, hd), dtype=torch.int8, device=DEV)
    expo = torch.empty((total, 2, Hkv, 16), dtype=torch.int8, device=DEV)
    lt, lc, le = _layer([n, n], Hkv, hd, 8, spare=0)
    places = np.array([3, (1 << 31) // each + 1, total - 1, total - 2, 0, (1 << 31) // each])
    dc, de = _device_layer(lc, le)
    codes[torch.as_tensor(places, device=DEV)], expo[torch.as_tensor(places, device=DEV)] = dc, de
    q = gen.normal(8, 13, (2, H * hd))
    out = torch.empty((2, H, hd), device=DEV)
    scratch = torch.empty(ld.ldk_attention_q8_scratch_bytes(2, H, Hkv, hd, n), dtype=torch.uint8, device=DEV)
    ld.ldk_paged_attention_q8(q.to(DEV), H * hd, codes, expo, _i32(places[lt]), _i32([0, 1]), _i32([n, n]), n, H, Hkv, hd, out, scratch)
    _check_decode(out, q, lt, lc, le, range(2), [n, n], H, Hkv, hd)
    tiles = _i32([[0, 1, n - 1, 0, 0, 0], [1, 1, n - 1, 1, 0, 0]])
    chunk = torch.empty((2, H, hd), device=DEV)
    scratch = torch.empty(ld.ldk_prefill_attention_q8_scratch_bytes(2, H, Hkv, hd, n), dtype=torch.uint8, device=DEV)
    ld.ldk_prefill_attention_q8(q.to(DEV), H * hd, codes, expo, _i32(places[lt]), tiles, H, Hkv, hd, chunk, n - 1, scratch=scratch)
    _check_prefill(chunk, q, lt, lc, le, tiles.tolist(), [n, n], H, Hkv, hd)
    pool = torch.zeros((6, 2, Hkv, 16, hd), dtype=torch.bfloat16, device=DEV)
    ranges = _i32([[0, 0, n], [1, 0, n]])
    ld.ldk_kv_from_q8(codes, expo, _i32(places[lt]), pool, _i32(lt), ranges, n, Hkv, hd)
    got = logical_pool(pool.cpu()).double().numpy()
    for s in range(2):
        k, v = _sequence(lt, lc, le, s, n)
        blocks = got[lt[s]].transpose(1, 0, 3, 2, 4).reshape(2, -1, Hkv, hd)[:, :n]
        assert np.array_equal(blocks[0], k) and np.array_equal(blocks[1], v)


# ---------------------------------------------------------------- prompt and chunk rows

def _run_prefill(q, rows, table, codes, expo, tiles, H, Hkv, hd, max_pos, window=0, cap=0.0, slopes=None, spare=0):
    dc, de = _device_layer(codes, expo)
    out = torch.full((rows, H, hd), 9.0, device=DEV)
    n = ld.ldk_prefill_attention_q8_scratch_bytes(len(tiles), H, Hkv, hd, max_pos, window)
    scratch = torch.full((n + spare,), 255, dtype=torch.uint8, device=DEV)
    ld.ldk_prefill_attention_q8(q.to(DEV), H * hd, dc, de, _i32(table), _i32(np.array(tiles)), H, Hkv, hd, out, max_pos, window=window, softcap=cap,
                                slopes=None if slopes is None else _f32(slopes), scratch=scratch)
    return out


def _check_prefill(out, q, table, codes, expo, tiles, lengths, H, Hkv, hd, window=0, cap=0.0, slopes=None, heads=None, some=None):
    """some: only every so many rows; heads: only these."""
    qd = q.double().numpy()
    got = out.double().cpu().numpy()
    for at, n, pos, s, first, prefix in tiles:
        k, v = _sequence(table, codes, expo, s, lengths[s])
        for r in range(0, n, some or 1):
            p = pos + r
            lo, hi = max(first, p - window + 1 if window else 0), max(p, prefix - 1)
            for h in heads or range(H):
                j = h // (H // Hkv)
                ref, bound = _attend(qd[at + r, h * hd:(h + 1) * hd], k[:, j], v[:, j], p, lo, hi, cap, float(np.float32(slopes[h])) if slopes is not None else 0.0,
                                     least=9)
                g = got[at + r, h]
                assert np.array_equal(np.isnan(g), np.isnan(ref)), (at, r, h)
                assert (np.abs(g - ref)[~np.isnan(ref)] <= bound[~np.isnan(ref)]).all(), (at, r, h, np.nanmax(np.abs(g - ref) / np.maximum(bound, 1e-300)))


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (128, 4, 1), (64, 3, 3), (64, 6, 2)])
@pytest.mark.parametrize("window,cap,bias", [(0, 0.0, False), (1, 0.0, False), (40, 10.0, False), (150, 0.0, True), (0, 30.0, True)])
def test_prefill_segments(hd, H, Hkv, window, cap, bias):
    """Chunks behind cached positions that begin and end anywhere, tiles of one row, of 128, and of less, prefixes and documents; gaps between the
    tiles' rows stay as they were."""
    # (rows, positions before, first visible, prefix) of each sequence
    segs = [(1, 0, 0, 0), (130, 0, 0, 0), (33, 100, 0, 0), (64, 37, 20, 0), (17, 300, 310, 0), (100, 63, 0, 120), (5, 15, 17, 19), (31, 129, 0, 31)]
    lengths = [b + n for n, b, _, _ in segs]
    table, codes, expo = _layer(lengths, Hkv, hd, hd + H + window)
    tiles, at = [], 3
    for s, (n, before, first, prefix) in enumerate(segs):
        for i in range(0, n, 128):
            tiles.append((at + i, min(128, n - i), before + i, s, first, prefix))
        at += n + s % 3
    q = gen.normal(window + H, 13, (at + 2, H * hd))
    kw = dict(window=window, cap=cap, slopes=_slopes(H) if bias else None)
    out = _run_prefill(q, at + 2, table, codes, expo, tiles, H, Hkv, hd, max(max(b + n, x) for (n, b, _, x) in segs) - 1, **kw)
    _check_prefill(out, q, table, codes, expo, tiles, lengths, H, Hkv, hd, **kw)
    named = np.zeros(at + 2, bool)
    for t in tiles:
        named[t[0]:t[0] + t[1]] = True
    assert (out[torch.as_tensor(~named)] == 9.0).all()


@pytest.mark.parametrize("hd,H,Hkv,n,before,window", [(128, 4, 4, 257, 1263, 0), (128, 4, 1, 64, 9000, 0), (128, 2, 2, 128, 20000, 0), (64, 2, 1, 130, 3900, 500),
                                                      (128, 4, 2, 1025, 0, 300), (128, 40, 40, 20, 2000, 0)])
def test_prefill_of_few_tiles_over_long_sequences(hd, H, Hkv, n, before, window):
    table, codes, expo = _layer([before + n], Hkv, hd, n)
    tiles = [(i, min(128, n - i), before + i, 0, 0, 0) for i in range(0, n, 128)]
    q = gen.normal(n, 13, (n, H * hd))
    out = _run_prefill(q, n, table, codes, expo, tiles, H, Hkv, hd, before + n - 1, window=window, spare=512)
    _check_prefill(out, q, table, codes, expo, tiles, [before + n], H, Hkv, hd, window=window, some=13, heads=sorted({0, H // 2, H - 1}))


def test_prefill_keeps_what_is_not_finite_where_it_is():
    H, Hkv, hd, n = 4, 2, 128, 150
    table, codes, expo = _layer([n, n], Hkv, hd, 9)
    expo[table[0, 4], 0, 1, 7] = -128      # the key of KV head 1 at position 71
    expo[table[1, 1], 1, 0, 2] = -128      # the value of KV head 0 at position 18
    q = gen.normal(9, 13, (2 * n, H * hd))
    q[10, 3] = float("nan")
    q[20, 2 * hd + 5] = float("inf")
    tiles = [(s * n + i, min(128, n - i), i, s, 0, 0) for s in range(2) for i in range(0, n, 128)]
    for window in (0, 30):
        out = _run_prefill(q, 2 * n, table, codes, expo, tiles, H, Hkv, hd, n - 1, window=window)
        _check_prefill(out, q, table, codes, expo, tiles, [n, n], H, Hkv, hd, window=window)


def test_prefill_of_units_of_any_size():
    H = Hkv = 2
    hd, n = 128, 140
    table, codes, expo = _layer([n], Hkv, hd, 10)
    expo[table[0, :8], 1] = gen.randint(10, 1, -40, 30, 8 * Hkv * 16).numpy().reshape(8, Hkv, 16)
    q = gen.normal(10, 13, (n, H * hd))
    q[::3] *= 1e-30
    q[1::5] *= 30.0
    q[7] = 0.0
    tiles = [(i, min(128, n - i), i, 0, 0, 0) for i in range(0, n, 128)]
    out = _run_prefill(q, n, table, codes, expo, tiles, H, Hkv, hd, n - 1)
    _check_prefill(out, q, table, codes, expo, tiles, [n], H, Hkv, hd)


# ---------------------------------------------------------------- together

def test_a_run_of_them_together():
    """A layer over the 8-bit cache as a model runs it: a prompt in two chunks, then decode steps of two sequences; every output against float64 on the
    cache's values.  Then one sequence moves into a bf16 pool, where the plain attention answers the same within its own tolerance."""
    H, Hkv, hd, rot = 8, 2, 128, 64
    lengths = [75, 40]
    table, total = _tables([96, 64], 12)
    codes, expo = np.zeros((total, 2, Hkv, 16, hd), np.int8), np.full((total, 2, Hkv, 16), -128, np.int8)
    dc, de = _device_layer(codes, expo)
    dt = _i32(table)
    gains = [gen.normal(12, 3 + i, (hd,), std=0.1, mean=1.0) for i in range(2)]
    width = (H + 2 * Hkv) * hd

    def append(pos, slot, stream):
        qkv = gen.normal(12, stream, (len(pos), width))
        cs = torch.empty((len(pos), rot // 2, 2), device=DEV)
        d = _i32(pos)
        ld.ldk_rope_table_scaled(d, rot, 10000.0, cs, factor=4.0, low=1.0, high=4.0, original=64, attention=1.1)
        q = torch.empty((len(pos), H * hd), device=DEV)
        ld.ldk_rope_kv_write_q8(qkv.to(DEV), cs, d, _i32(slot), dt, dc, de, H, Hkv, hd, q, rot=rot, interleaved=True, q_gain=gains[0].to(DEV),
                                k_gain=gains[1].to(DEV), eps=1e-6)
        _append_reference(qkv, pos, slot, table, cs.cpu(), H, Hkv, hd, rot, True, *gains, 1e-6, codes, expo)
        return q

    for s, n in enumerate(lengths):
        for a, b in ((0, 33), (33, n)):
            q = append(list(range(a, b)), [s] * (b - a), 20 + s * 2 + (a > 0))
            tiles = [(0, b - a, a, s, 0, 0)]
            out = torch.full((b - a, H, hd), 9.0, device=DEV)
            scratch = torch.empty(ld.ldk_prefill_attention_q8_scratch_bytes(1, H, Hkv, hd, b - 1), dtype=torch.uint8, device=DEV)
            ld.ldk_prefill_attention_q8(q, H * hd, dc, de, dt, _i32(tiles), H, Hkv, hd, out, b - 1, scratch=scratch)
            assert np.array_equal(_logical(dc, de)[0], codes) and np.array_equal(de.cpu().numpy(), expo)
            _check_prefill(out, q.cpu(), table, codes, expo, tiles, {s: b}, H, Hkv, hd)
    ctx = list(lengths)
    for step in range(3):
        q = append(ctx, [0, 1], 40 + step)
        ctx = [c + 1 for c in ctx]
        out = torch.full((2, H, hd), 9.0, device=DEV)
        scratch = torch.empty(ld.ldk_attention_q8_scratch_bytes(2, H, Hkv, hd, max(ctx)), dtype=torch.uint8, device=DEV)
        ld.ldk_paged_attention_q8(q, H * hd, dc, de, dt, _i32([0, 1]), _i32(ctx), max(ctx), H, Hkv, hd, out, scratch)
        _check_decode(out, q.cpu(), table, codes, expo, [0, 1], ctx, H, Hkv, hd)
    pool = torch.full((total, 2, Hkv, 16, hd), float("nan"), dtype=torch.bfloat16, device=DEV)
    ld.ldk_kv_from_q8(dc, de, dt, pool, dt, _i32([[0, 0, ctx[0]]]), ctx[0], Hkv, hd)
    plain = torch.empty((1, H, hd), device=DEV)
    scratch = torch.empty(ld.ldk_attention_scratch_bytes(1, H, Hkv, hd, ctx[0]), dtype=torch.uint8, device=DEV)
    ld.ldk_paged_attention(q[:1], H * hd, pool, dt, _i32([0]), _i32(ctx[:1]), ctx[0], H, Hkv, hd, plain, scratch)
    # the plain kernel holds queries and probabilities in 16 bits
    assert (plain - out[:1]).norm().item() <= 1e-4 * out[:1].norm().item()


def test_recorded_steps_and_other_streams():
    """Angles, append and both attentions in a graph on a side stream; two graphs over the same scratch; every replay, with new inputs and other work
    between, gives what the calls give one by one."""
    H, Hkv, hd, T = 8, 2, 128, 3
    lengths = [700, 90, 333]
    table, codes, expo = _layer([n + 40 for n in lengths], Hkv, hd, 14)
    dc, de = _device_layer(codes, expo)
    dt, slot = _i32(table), _i32(range(T))
    qkv = torch.empty((T, (H + 2 * Hkv) * hd), device=DEV)
    pos, ctx = _i32(lengths), _i32([n + 1 for n in lengths])
    tiles = _i32([(t, 1, n, t, 0, 0) for t, n in enumerate(lengths)])
    q, cs = torch.empty((T, H * hd), device=DEV), torch.empty((T, hd // 2, 2), device=DEV)
    most = max(lengths) + 40
    a, b = torch.empty((T, H, hd), device=DEV), torch.empty((T, H, hd), device=DEV)
    scratch = torch.empty(max(16, ld.ldk_attention_q8_scratch_bytes(T, H, Hkv, hd, most), ld.ldk_prefill_attention_q8_scratch_bytes(T, H, Hkv, hd, most)),
                          dtype=torch.uint8, device=DEV)

    def step():
        ld.ldk_rope_table_scaled(pos, hd, 10000.0, cs)
        ld.ldk_rope_kv_write_q8(qkv, cs, pos, slot, dt, dc, de, H, Hkv, hd, q)
        ld.ldk_paged_attention_q8(q, H * hd, dc, de, dt, slot, ctx, most, H, Hkv, hd, a, scratch)
        ld.ldk_prefill_attention_q8(q, H * hd, dc, de, dt, tiles, H, Hkv, hd, b, most, scratch=scratch)

    side = torch.cuda.Stream()
    graphs = []
    for _ in range(2):
        qkv.normal_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
        graphs.append(g)
    for i in range(4):
        qkv.copy_(gen.normal(30 + i, 1, tuple(qkv.shape)).to(DEV))
        pos.copy_(_i32([n + i for n in lengths]))
        ctx.copy_(_i32([n + i + 1 for n in lengths]))
        tiles.copy_(_i32([(t, 1, n + i, t, 0, 0) for t, n in enumerate(lengths)]))
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (q, a, b, dc, de)]
        for x in (q, a, b):
            x.fill_(5.0)
        step()
        assert all(torch.equal(x, y) for x, y in zip(got, (q, a, b, dc, de)))
        assert (a - b).norm().item() <= 4e-6 * b.norm().item()      # two kernels, the same rows


def test_one_tensor_in_host_memory_is_refused():
    """Each tensor of each call in turn; a refused call launches nothing."""
    H = Hkv = 2
    hd = 64
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device=DEV)      # noqa: E731
    codes, expo, table = z(1, 2, Hkv, 16, hd, dtype=torch.int8), z(1, 2, Hkv, 16, dtype=torch.int8), z(1, 1, dtype=torch.int32)
    i1, gain, scratch = z(1, dtype=torch.int32), z(hd), z(1 << 20)
    pool, ranges, tiles, q, out, slopes = z(1, 2, Hkv, 16, hd), z(1, 3, dtype=torch.int32), z(1, 6, dtype=torch.int32), z(1, H * hd), z(1, H, hd), z(H)
    calls = [(ld.ldk_rope_table_scaled, (i1, hd, 1e4, z(1, hd // 2, 2)), {}),
             (ld.ldk_rope_kv_write_q8, (z(1, 3 * H * hd), z(1, hd // 2, 2), i1, i1, table, codes, expo, H, Hkv, hd, q), dict(q_gain=gain, k_gain=gain)),
             (ld.ldk_kv_to_q8, (pool, table, codes, expo, table, ranges, 1, Hkv, hd), {}),
             (ld.ldk_kv_from_q8, (codes, expo, table, pool, table, ranges, 1, Hkv, hd), {}),
             (ld.ldk_paged_attention_q8, (q, H * hd, codes, expo, table, i1, i1, 1, H, Hkv, hd, out, scratch), dict(first=i1, slopes=slopes)),
             (ld.ldk_prefill_attention_q8, (q, H * hd, codes, expo, table, tiles, H, Hkv, hd, out, 0), dict(scratch=scratch, slopes=slopes))]
    for call, args, more in calls:
        call(*args, **more)
        for i, t in enumerate(args):
            if isinstance(t, torch.Tensor):
                with pytest.raises(ld.LdError, match="device"):
                    call(*args[:i], t.cpu(), *args[i + 1:], **more)
        for name, t in more.items():
            with pytest.raises(ld.LdError, match="device"):
                call(*args, **{**more, name: t.cpu()})
    torch.cuda.synchronize()


def test_tensors_in_host_memory_are_refused():
    H = Hkv = 2
    hd = 64
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)      # noqa: E731
    codes, expo, table = z(1, 2, Hkv, 16, hd, dtype=torch.int8), z(1, 2, Hkv, 16, dtype=torch.int8), z(1, 1, dtype=torch.int32)
    i1, scratch = z(1, dtype=torch.int32), z(1 << 20)
    torch.cuda.current_stream()
    calls = [lambda: ld.ldk_rope_kv_write_q8(z(1, 3 * H * hd), z(1, hd // 2, 2), i1, i1, table, codes, expo, H, Hkv, hd, z(1, H * hd)),
             lambda: ld.ldk_kv_to_q8(z(1, 2, Hkv, 16, hd), table, codes, expo, table, z(1, 3, dtype=torch.int32), 1, Hkv, hd),
             lambda: ld.ldk_kv_from_q8(codes, expo, table, z(1, 2, Hkv, 16, hd), table, z(1, 3, dtype=torch.int32), 1, Hkv, hd),
             lambda: ld.ldk_paged_attention_q8(z(1, H * hd), H * hd, codes, expo, table, i1, i1, 1, H, Hkv, hd, z(1, H, hd), scratch),
             lambda: ld.ldk_prefill_attention_q8(z(1, H * hd), H * hd, codes, expo, table, z(1, 6, dtype=torch.int32), H, Hkv, hd, z(1, H, hd), 0, scratch=scratch)]
    torch.zeros(1, device=DEV)      # the GPU is up
    for call in calls:
        with pytest.raises(ld.LdError) as e:
            call()
        assert e.value.status == ld.LD_E_INVAL and "device" in str(e.value)


@pytest.mark.parametrize("G", [1, 3, 16])
def test_unmapped_blocks_inside_a_sequence_are_not_seen(G):
    """Positions whose block the table does not map take no part, in both attention calls; neither do positions beyond the table."""
    Hkv, hd, n = 2, 128, 300
    H = G * Hkv
    table, codes, expo = _layer([n], Hkv, hd, 15)
    table[0, [0, 4, 5, 11]] = -1
    kept = np.array([p for p in range(n) if table[0, p // 16] >= 0])
    q = gen.normal(15, 13, (1, H * hd))
    full = table.copy()
    full[0, table[0] < 0] = 0      # for reading the values: these positions are dropped below
    k, v = _sequence(full, codes, expo, 0, n)
    for width, wide in ((19, n), (15, 240)):      # the second table ends at position 240
        cut = np.ascontiguousarray(table[:, :width])
        out = _run_decode(q, cut, codes, expo, [0], [n], H, Hkv, hd)
        chunk = _run_prefill(q, 1, cut, codes, expo, [(0, 1, n - 1, 0, 0, 0)], H, Hkv, hd, n - 1)
        use = kept[kept < wide]
        for h in range(H):
            ref, bound = _attend(q[0, h * hd:(h + 1) * hd].double().numpy(), k[use, h // G], v[use, h // G], 0, 0, len(use) - 1, 0.0, 0.0, least=9)
            for got in (out, chunk):
                assert (np.abs(got[0, h].double().cpu().numpy() - ref) <= bound).all()


def test_two_streams_at_once():
    """Calls on two streams over one cache, each with its own scratch, give what they give alone."""
    H, Hkv, hd, n = 8, 2, 128, 5000
    table, codes, expo = _layer([n, n - 7], Hkv, hd, 16)
    dc, de = _device_layer(codes, expo)
    dt = _i32(table)
    qs = [gen.normal(16, 20 + i, (2, H * hd)).to(DEV) for i in range(2)]
    size = ld.ldk_attention_q8_scratch_bytes(2, H, Hkv, hd, n)

    def call(q, out, scratch, stream):
        ld.ldk_paged_attention_q8(q, H * hd, dc, de, dt, _ctx[0], _ctx[1], n, H, Hkv, hd, out, scratch, stream=stream)

    _ctx = _i32([0, 1]), _i32([n, n - 7])
    alone = []
    for q in qs:
        alone.append(torch.empty((2, H, hd), device=DEV))
        call(q, alone[-1], torch.empty(size, dtype=torch.uint8, device=DEV), None)
    torch.cuda.synchronize()
    streams, outs, scratch = [torch.cuda.Stream() for _ in qs], [torch.zeros((2, H, hd), device=DEV) for _ in qs], [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for q, o, s, st in zip(qs, outs, scratch, streams):
            call(q, o, s, st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))


@pytest.mark.parametrize("hd,H,Hkv", [(128, 4, 4), (64, 8, 2)])
def test_empty_calls_and_padded_tiles(hd, H, Hkv):
    """No rows, no tiles; tiles of no rows beside others; a batch in which no row sees anything."""
    table, codes, expo = _layer([20, 30], Hkv, hd, 17)
    none = torch.empty((0, H * hd), device=DEV)
    assert _run_decode(none, table, codes, expo, [], [], H, Hkv, hd, max_ctx=0).shape[0] == 0
    out = _run_decode(gen.normal(17, 1, (2, H * hd)), table, codes, expo, [0, 1], [0, 0], H, Hkv, hd, max_ctx=0)
    assert (out == 0).all()
    q = gen.normal(17, 2, (8, H * hd))
    tiles = [(0, 0, 0, 0, 0, 0), (3, 4, 16, 0, 0, 0), (0, 0, 0, -1, 0, 0), (0, 2, 5, 1, 0, 0)]
    out = _run_prefill(q, 8, table, codes, expo, tiles, H, Hkv, hd, 19)
    _check_prefill(out, q, table, codes, expo, tiles, [20, 30], H, Hkv, hd)
    assert (out[[2, 7]] == 9.0).all()
    ld.ldk_prefill_attention_q8(q.to(DEV), H * hd, *_device_layer(codes, expo), _i32(table), torch.empty((0, 6), dtype=torch.int32, device=DEV), H, Hkv, hd, out, 0,
                                scratch=torch.empty(16, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("hd,H,Hkv", [(128, 2, 2), (64, 4, 1)])
def test_keys_and_values_near_the_ends_of_their_range(hd, H, Hkv):
    """Keys up to 2^120 under queries of 2^-115, and keys of 2^-120 and 2^-104 under queries of 2^108; values over 2^84, zeros first."""
    n = 150
    for keys, small in (((113, 100, 90), -115), ((-126, -124, -110), 108)):
        table, codes, expo = _layer([n], Hkv, hd, 18)
        pick = gen.randint(18, 1, 0, len(keys) - 1, 10 * Hkv * 16).numpy().reshape(10, Hkv, 16)
        expo[table[0, :10], 0] = np.array(keys)[pick]
        expo[table[0, :10], 1] = gen.randint(18, 2, -42, 42, 10 * Hkv * 16).numpy().reshape(10, Hkv, 16)
        codes[table[0, :4], 1] = 0
        expo[table[0, :4], 1] = -126
        q = (gen.normal(18, 13, (n, H * hd)).double() * 2.0 ** small).float()
        tiles = [(i, min(128, n - i), i, 0, 0, 0) for i in range(0, n, 128)]
        out = _run_prefill(q, n, table, codes, expo, tiles, H, Hkv, hd, n - 1)
        _check_prefill(out, q, table, codes, expo, tiles, [n], H, Hkv, hd)
        rows = [0, 63, 64, 149]
        out = _run_decode(q[rows].contiguous(), table, codes, expo, [0] * 4, [r + 1 for r in rows], H, Hkv, hd)
        _check_decode(out, q[rows].contiguous(), table, codes, expo, [0] * 4, [r + 1 for r in rows], H, Hkv, hd)


def test_appends_and_moves_to_blocks_past_two_and_four_gigabytes():
    """Few and many rows, and a range moved: what lands in blocks whose bytes begin past 2^31 and 2^32 is what lands in a pool of four blocks."""
    H = Hkv = 32
    hd, n = 128, 60
    each = 2 * Hkv * 16 * hd
    total = (1 << 32) // each + 5
    places = np.array([total - 1, (1 << 31) // each + 1, total - 3, 1], np.int32)
    far = torch.empty((total, 2, Hkv, 16, hd), dtype=torch.int8, device=DEV), torch.empty((total, 2, Hkv, 16), dtype=torch.int8, device=DEV)
    near = torch.zeros((4, 2, Hkv, 16, hd), dtype=torch.int8, device=DEV), torch.zeros((4, 2, Hkv, 16), dtype=torch.int8, device=DEV)
    at = torch.as_tensor(places, device=DEV).long()
    far_table, near_table = _i32(places[None]), _i32([[0, 1, 2, 3]])
    cos_sin = torch.empty((n, hd // 2, 2), device=DEV)
    ld.ldk_rope_table_scaled(_i32(np.arange(n)), hd, 1e4, cos_sin)
    pool = gen.normal(19, 3, (4, 2, Hkv, 16, hd)).to(torch.bfloat16).to(DEV)
    for pos in ([5, 59], list(range(n)), None):
        for (codes, expo), table in ((far, far_table), (near, near_table)):
            if pos is None:
                ld.ldk_kv_to_q8(pool, near_table, codes, expo, table, _i32([[0, 1, n - 1]]), n, Hkv, hd)
                continue
            qkv = gen.normal(19, len(pos), (len(pos), 3 * H * hd)).to(DEV)
            ld.ldk_rope_kv_write_q8(qkv, cos_sin[pos].contiguous(), _i32(pos), _i32([0] * len(pos)), table, codes, expo, H, Hkv, hd, torch.empty((len(pos), H * hd), device=DEV))
        slots = [5, 59] if pos == [5, 59] else list(range(n))
        for p in slots:
            b, i = p // 16, p % 16
            assert torch.equal(far[1][at[b], :, :, i], near[1][b, :, :, i])
            assert torch.equal(far[0][at[b], 0, :, i], near[0][b, 0, :, i])
            a, c = (x.view(Hkv, hd, 16)[:, :, i] for x in (far[0][at[b], 1], near[0][b, 1]))
            assert torch.equal(a, c)
