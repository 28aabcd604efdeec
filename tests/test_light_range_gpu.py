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
