"""4-bit linear layers on rows with columns of very unlike size, as the input of a down projection has them."""
import pytest
import torch

from workloads import gen
from test_light_ops_gpu import _linear, _packed, _rel, _w4

pytestmark = pytest.mark.gpu

FORMS = [(32, True, torch.bfloat16), (32, False, torch.float32), (64, True, torch.float32), (64, False, torch.bfloat16), (128, True, torch.bfloat16),
         (128, True, torch.float32), (128, False, torch.bfloat16)]
OUT = (5, 166, 519)      # columns: one in each half of the four that a thread splits, in three tiles of 128


def _case(T, group, zeros, scales):
    """A matrix whose columns OUT are all zero (their codes are the zero points), 640 columns."""
    N, K = 72, 640
    c, s, z, _ = _w4(T + group, N, K, group, zeros, scales)
    col = torch.arange(K) // group
    zero = z[:, col] if zeros else torch.full_like(c, 8)
    for k in OUT:
        c[:, k] = zero[:, k]
    W = (c - zero).double() * s.double()[:, col]
    return c, s, z, W, N, K


@pytest.mark.parametrize("group,zeros,scales", FORMS)
@pytest.mark.parametrize("T", [1, 2, 6, 30, 150])
def test_a_column_without_weight_leaves_nothing(T, group, zeros, scales):
    """Small whole numbers beside columns some 10^4 times as large whose weights are zero: the whole numbers are exact in the operands, so that nothing
    but float32's rounding of the groups' sums remains: at most one half of 2^-23 for each of the product with the scale and the sum, over up to 20
    groups of random sign, of totals that are no larger than the mass."""
    c, s, z, W, N, K = _case(T, group, zeros, scales)
    x = gen.randint(T, 5, -7, 7, T * K).view(T, K).float()
    for i, k in enumerate(OUT):
        x[:, k] = (gen.uniform01(T, 6 + i, 0, T) + 1.0) * 20000.0
    y = _linear(_packed(c, s, z, N, K, group), x).cpu().double()
    ref = x.double() @ W.t()
    assert ((y - ref).abs() <= 2.0 ** -23 * 20 * (x.double().abs() @ W.abs().t())).all()
    assert _rel(y, ref) <= 1e-6


@pytest.mark.parametrize("group,zeros,scales", FORMS)
@pytest.mark.parametrize("factor", [1.0, 300.0, 3e4, 3e6, 1e9])
@pytest.mark.parametrize("T", [1, 2, 30, 150])
def test_what_a_column_keeps(T, factor, group, zeros, scales):
    """The bound that the header states for what a column loses: 2^-22 of the largest of its 128 columns, 2^-25 where it is below a quarter of that, never more than
    2^-11 of itself, and on top 2^-35 of the row's largest (what the smallest fp16 number leaves).  Every loss at its worst and in the same direction; the
    sums' roundings as in the test of odd shapes, on what is left when the columns without weight are taken out."""
    c, s, z, W, N, K = _case(T, group, zeros, scales)
    x = gen.normal(T, 5, (T, K))
    x[:, 5] *= factor      # one column; the other tiles of 128 have none
    x = x.contiguous()
    y = _linear(_packed(c, s, z, N, K, group), x).cpu().double()
    xd = x.double()
    most = xd.abs().view(T, K // 128, 128).amax(2).repeat_interleave(128, 1)
    lost = torch.minimum(torch.where(xd.abs() < most / 4, 2.0 ** -25, 2.0 ** -22) * most, 2.0 ** -11 * xd.abs()) + 2.0 ** -35 * xd.abs().amax(1, keepdim=True)
    some = torch.where(W.abs().sum(0) > 0, xd.abs(), 0.0)
    mass = some @ (W.abs() + 8 * s.double()[:, torch.arange(K) // group]).t()
    # the lo terms' sums are float32's too: up to 15 times 2.5 quanta of 2^-12 of the tile's largest a column, 2^-24 of that at each of four steps
    rounding = 2.0 ** -23 * (60 + K / 32) * mass + 2.0 ** -24 * 4 * 15 * 2.5 * 2.0 ** -12 * most.sum(1, keepdim=True) * s.double().amax(1)
    assert ((y - xd @ W.t()).abs() <= lost @ W.abs().t() + rounding).all()
