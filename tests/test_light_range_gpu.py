"""Block-sparse attention at the ends of the number range: scores beyond float32 on the way, keys and values that are not finite, and sums whose terms
cancel, against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2406_00059_amd as ld
from test_light_ops_gpu import ATTENTION, _rel, _run_sparse, _sparse64, _sparse_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("blocks", [40, 700], ids=["one-launch", "two-launches"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("q_exp,k_exp", [(116, -60), (-60, 100), (-120, 100), (100, -100)])
def test_choice_between_queries_and_keys_of_unlike_magnitude(dtype, blocks, q_exp, k_exp):
    """A score is the sum times both powers of two: neither alone takes it out of the range.  Queries up to 2^118 with keys around 2^-60."""
    H, Hkv, hd, ctx, budget = 4, 2, 128, [16 * blocks - 3], 9
    q, logical, table, slot = _sparse_case(101, dtype, H, Hkv, hd, ctx)
    q = q * 2.0 ** q_exp
    logical = logical.clone()
    logical[:, 0] *= 2.0 ** k_exp
    out, sel, bounds, unit = _run_sparse(q, logical, table, slot, ctx, H, Hkv, hd, 0, budget, 1, 2)
    _, want = _sparse64(q.numpy(), logical.double().numpy(), bounds, unit, table, slot, ctx, H, Hkv, hd, 0, budget, 1, 2)
    np.testing.assert_array_equal(sel.cpu().numpy(), want)


SHAPES = [(4, 2, 128, torch.bfloat16), (8, 1, 128, torch.bfloat16), (3, 3, 64, torch.bfloat16), (2, 1, 64, torch.float32), (20, 2, 128, torch.bfloat16)]


@pytest.mark.parametrize("blocks,window", [(40, 0), (700, 0), (40, 300), (6, 0)], ids=["one-launch", "two-launches", "band", "all-blocks"])
@pytest.mark.parametrize("H,Hkv,hd,dtype", SHAPES)
def test_keys_and_values_that_are_infinite(H, Hkv, hd, dtype, blocks, window):
    """A key whose product with a query is -infinity has no weight, also where it is the first or the only one of its block; an infinite value
    makes its own dimension infinite and no other; heads of other rows and other KV heads are as they would be without."""
    ctx, budget, first, last = [16 * blocks - 3, 16 * blocks - 15, 1, 90], 9, 1, 2
    q, logical, table, slot = _sparse_case(102, dtype, H, Hkv, hd, ctx)
    q[:, :, 7] = q[:, :, 7].abs() + 0.25
    logical = logical.clone()
    low = lambda t, b: table[slot[t], b]
    for b in (blocks - 1, blocks - 2, 0, blocks - 4):
        logical[low(0, b), 0, 0, 3, 7] = -float("inf")
    logical[low(1, blocks - 1), 0, 0, 0, 7] = -float("inf")        # the only position of its block
    logical[low(1, blocks - 2), 0, 0, :, 7] = -float("inf")        # all positions
    logical[low(3, 2), 1, 0, 5, 11] = float("inf")
    logical[low(3, 5), 1, 0, 1, 12] = -float("inf")
    args = (table, slot, ctx, H, Hkv, hd, window, budget, first, last)
    out, sel, bounds, unit = _run_sparse(q, logical, *args)
    with np.errstate(invalid="ignore"):
        ref, want = _sparse64(q.numpy(), logical.double().numpy(), bounds, unit, *args)
    np.testing.assert_array_equal(sel.cpu().numpy(), want)
    out = out.cpu().double()
    ref = torch.from_numpy(ref)
    assert not torch.isnan(ref).any() and torch.isinf(ref[3, 0, 11:13]).all()
    assert torch.equal(torch.isinf(out), torch.isinf(ref)) and torch.equal(out[torch.isinf(out)], ref[torch.isinf(ref)])
    assert _rel(out[torch.isfinite(ref)], ref[torch.isfinite(ref)]) <= ATTENTION


@pytest.mark.parametrize("H,Hkv,hd,dtype", SHAPES)
def test_a_row_whose_only_key_has_no_weight_is_nan(H, Hkv, hd, dtype):
    """As the quotient of the definition, 0 / 0; the row beside it is not touched."""
    q, logical, table, slot = _sparse_case(103, dtype, H, Hkv, hd, [1, 50])
    q[:, :, 7] = q[:, :, 7].abs() + 0.25
    logical = logical.clone()
    logical[table[slot[0], 0], 0, :, 0, 7] = -float("inf")
    args = (table, slot, [1, 50], H, Hkv, hd, 0, 4, 1, 1)
    out, sel, bounds, unit = _run_sparse(q, logical, *args)
    with np.errstate(invalid="ignore"):
        ref, want = _sparse64(q.numpy(), logical.double().numpy(), bounds, unit, *args)
    np.testing.assert_array_equal(sel.cpu().numpy(), want)
    assert torch.isnan(out[0]).all() and np.isnan(ref[0]).all() and _rel(out[1], torch.from_numpy(ref[1])) <= ATTENTION


def _bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).bfloat16().float().numpy()


def _third(x):
    """What is left of float32 numbers behind two bf16 terms, and the two terms' sum."""
    x = np.asarray(x, np.float32)
    a = _bf16(x)
    b = _bf16(x - a)
    return (x - a) - b, a.astype(np.float64) + b


@pytest.mark.parametrize("H,Hkv,hd", [(1, 1, 128), (2, 2, 64), (8, 1, 128), (6, 1, 64)])
@pytest.mark.parametrize("blocks", [24, 700], ids=["one-launch", "two-launches"])
def test_queries_keep_their_last_bits(H, Hkv, hd, blocks):
    """Keys whose products with a query cancel while those with its bits behind the 16th add up.  A score is held to five roundings of 2^-23 of the
    products' mass: up to four steps of 32 dimensions, each of which may cut 2^-23 of a partial sum of half the mass twice, and the query's scaling.
    A query of two bf16 terms would be off by more than twice that, which the oracle with such queries shows."""
    ctx = [16 * blocks - 3]
    q, logical, table, slot = _sparse_case(104, torch.bfloat16, H, Hkv, hd, ctx)
    scale = np.float32(np.float32(1.4426950408889634) / np.sqrt(np.float32(hd)))
    q = (1.0 + q.abs() * 0.2) * q.sign()
    q[0, 1:] = q[0, 0]      # one query: the keys are made for it
    rest, two = _third(q[0, 0].numpy() * scale)
    u = np.sign(rest) + (rest == 0)
    side = q[0, 0].numpy() * u > 0
    u[side] *= np.abs(q[0, 0].numpy()[~side]).sum() / np.abs(q[0, 0].numpy()[side]).sum()
    sign = torch.where(torch.arange(16) % 2 == 0, 1.0, -1.0)
    logical = logical.clone()
    logical[:, 0] = (torch.from_numpy(u).float() * 16 * sign[:, None]).bfloat16()
    logical[:, 1] = sign[:, None].bfloat16()
    args = (table, slot, ctx, H, Hkv, hd, 0, 9, 1, 2)
    out, sel, bounds, unit = _run_sparse(q, logical, *args)
    keys = logical.double().numpy()
    ref, want = _sparse64(q.numpy(), keys, bounds, unit, *args)
    np.testing.assert_array_equal(sel.cpu().numpy(), want)
    mass = np.abs(q[0, 0].double().numpy()) @ np.abs(keys[0, 0, 0, 0]) / np.sqrt(hd)
    tol = 2.0 ** -23 * 5 * mass      # of the result too: two groups of positions whose scores are off in opposite directions weigh +1 and -1
    planted = np.broadcast_to(two / (1.4426950408889634 / np.sqrt(hd)), (1, H, hd))
    wrong, same = _sparse64(planted, keys, bounds, unit, *args)
    np.testing.assert_array_equal(same, want)
    assert np.abs(wrong - ref).min() > 2 * tol
    assert np.abs(out.cpu().double().numpy() - ref).max() <= tol


@pytest.mark.parametrize("H,Hkv,hd", [(1, 1, 128), (2, 2, 64), (8, 1, 128), (6, 1, 64)])
@pytest.mark.parametrize("blocks", [24, 700], ids=["one-launch", "two-launches"])
def test_probabilities_keep_their_last_bits(H, Hkv, hd, blocks):
    """One position of a block has the maximum, the other fifteen a probability with a long third term; the values cancel.  The result is held to
    eight roundings of 2^-23 of the values' mass; probabilities of two bf16 terms are off by more than twice that."""
    ctx = [16 * blocks]
    q, logical, table, slot = _sparse_case(105, torch.bfloat16, H, Hkv, hd, ctx)
    q[:] = 0
    q[..., 0] = 1
    steps = np.arange(1, 200) / 16.0      # differences of the first key entry: exact in bf16
    p = np.exp(-steps / np.sqrt(hd))
    rest, _ = _third(p)
    best = int(np.argmax(np.abs(rest) / p))
    d, p, rest = steps[best], p[best], rest[best]
    logical = logical.clone()
    logical[:, 0] = 0
    logical[:, 0, :, 1:, 0] = -d
    low = float(torch.tensor(15 * p * 32).bfloat16())
    logical[:, 1] = 32.0
    logical[:, 1, :, 0] = -low
    args = (table, slot, ctx, H, Hkv, hd, 0, 9, 1, 2)
    out, sel, bounds, unit = _run_sparse(q, logical, *args)
    ref, want = _sparse64(q.numpy(), logical.double().numpy(), bounds, unit, *args)
    np.testing.assert_array_equal(sel.cpu().numpy(), want)
    total = 1 + 15 * p
    tol = 2.0 ** -23 * 8 * (low + 15 * p * 32) / total
    assert abs(15 * rest * 32 / total) > 2 * tol
    assert np.abs(out.cpu().double().numpy() - ref).max() <= tol
