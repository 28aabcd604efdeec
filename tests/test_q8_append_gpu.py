"""What a row appends to the 8-bit cache does not depend on how many rows its call has."""
import numpy as np
import pytest
import torch

import paper_2406_00059_amd as ld
from workloads import gen
from test_q8_gpu import DEV, _device_layer, _i32

pytestmark = pytest.mark.gpu


def _border_rows(n, hd, seed):
    """Rows [n, hd] whose mean square is 1 to within some 2^-52, by three last elements that make it up, and which hold 65.5 / 32 and 64.5 / 32: under a norm
    without gains these lie on the border of two codes, on either side of it with the last bit of the sum of squares."""
    rs = np.random.RandomState(seed)
    rows = []
    while len(rows) < n:
        x = rs.normal(size=hd).astype(np.float32).clip(-1.9, 1.9)
        x[3], x[hd // 2 + 1] = 65.5 / 32, -64.5 / 32
        fill = rs.choice([i for i in range(hd) if i not in (3, hd // 2 + 1)], 3, replace=False)
        x[fill] = 0
        x *= np.where((np.arange(hd) == 3) | (np.arange(hd) == hd // 2 + 1), 1, np.float32(0.93))
        for i in fill:
            rest = hd - (x.astype(np.float64) ** 2).sum()
            x[i] = np.sqrt(max(rest, 0.0)) * (1 - 2.0 ** -24)
        if np.abs(x).max() < 3.9 and abs(hd - (x.astype(np.float64) ** 2).sum()) < hd * 2.0 ** -50:
            rows.append(x)
    return torch.as_tensor(np.stack(rows))


@pytest.mark.parametrize("hd,H,Hkv", [(64, 2, 1), (128, 2, 2)])
@pytest.mark.parametrize("rot,interleaved", [("none", False), ("all", False), ("all", True), ("half", False), ("half", True)])
@pytest.mark.parametrize("sizes", [(1, 7), (47,)])
def test_codes_do_not_depend_on_the_number_of_rows(hd, H, Hkv, rot, interleaved, sizes):
    rot = {"none": 0, "all": hd, "half": hd // 2}[rot]
    T = 240
    qkv = torch.cat([_border_rows(T, hd, i) for i in range(H + Hkv)] + [gen.normal(1, 2, (T, Hkv * hd))], 1).contiguous()
    cos_sin = None
    if rot:      # turns by nothing, so that the borders stay, and by any angle
        angle = gen.normal(2, 2, (T, rot // 2)).double() * (torch.arange(T) % 2)[:, None]
        cos_sin = torch.stack([torch.cos(angle), torch.sin(angle)], -1).float().to(DEV)
    table = _i32(np.arange(15)[None])
    ones = torch.ones(hd, device=DEV)
    got = []
    for parts in [(T,)] + [(n,) for n in sizes]:
        dc, de = _device_layer(np.zeros((15, 2, Hkv, 16, hd), np.int8), np.zeros((15, 2, Hkv, 16), np.int8))
        q = torch.empty((T, H * hd), device=DEV)
        for a in range(0, T, parts[0]):
            b = min(a + parts[0], T)
            cs = cos_sin[a:b].contiguous() if rot else None
            ld.ldk_rope_kv_write_q8(qkv[a:b].to(DEV), cs, _i32(np.arange(a, b)), _i32([0] * (b - a)), table, dc, de, H, Hkv, hd, q[a:b], rot=rot,
                                    interleaved=interleaved, q_gain=ones, k_gain=ones, eps=0.0)
        got.append((dc, de, q))
    for other in got[1:]:
        assert all(torch.equal(x, y) for x, y in zip(got[0], other)), [(x != y).sum().item() for x, y in zip(got[0], other)]
