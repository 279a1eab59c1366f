"""Rounding of kept rows to 4 bits where it decides: halfway cases and their neighbours, the ends of the exponents (exact: the same bytes)."""
import numpy as np
import pytest
import torch

from oracle import kept_oracle as ko
from paper_2510_20787_amd import binding as B
from tests.kept_util import f64, kept_values

pytestmark = pytest.mark.gpu

HALFWAY = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)


def rows_of(dtype, D):
    """Rows whose groups have a given largest magnitude and hold every halfway quotient, one step below and one above it."""
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    step = torch.finfo(td).eps
    rows = []
    for k in (-126, -121, -120, -119, -118, -60, -3, 0, 1, 90, 125, 126, 127):
        for m in (1.0, 1.0 + step, 1.5, 1.75 - step, 1.75, 1.75 + step, 2.0 - step):
            top = torch.tensor(m * 2.0 ** k, dtype=torch.float64)
            E = k - 2 if m <= 1.75 or k == 127 else k - 1
            near = [h * 2.0 ** E * f for h in HALFWAY for f in (1.0 - step / 2, 1.0, 1.0 + step)]
            near = torch.tensor([x for x in near if x <= float(top)], dtype=torch.float64)
            for sign in (1.0, -1.0):
                row = torch.zeros(D, dtype=torch.float64)
                row[:len(near)] = sign * near
                row[31] = -sign * top
                row[32:64] = row[:32].flip(0)
                row[64:] = -row[:64].repeat(D // 64 - 1) if D > 64 else row[64:]
                rows.append(row)
    return torch.stack(rows).to(td)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_halfway_quotients(dtype, D):
    rows = rows_of(dtype, D)
    assert bool(torch.isfinite(rows.float()).all())
    cfg = B.make_cfg(1, 1, D, 4, len(rows), 0, 0.0, 0.0, dtype)
    cache = B.alloc_cache(cfg, 1)
    cache.k_ret[0, 0] = rows.cuda()
    cache.v_ret[0, 0] = rows.flip(0).cuda()
    cache.ret_count.fill_(len(rows))
    packed = B.ltea_kept_pack(cfg, cache)
    back = B.alloc_cache(cfg, 1)
    back.ret_count.copy_(cache.ret_count)
    B.ltea_kept_unpack(cfg, packed, back)
    blocks = packed[0, 0].cpu().numpy()
    for i in range(blocks.shape[0]):
        kc, vc, ke, ve = ko.read_block(blocks[i], D)
        for codes, byte, src in ((kc, ke, cache.k_ret), (vc, ve, cache.v_ret)):
            want = ko.encode(f64(src[0, 0, 32 * i:32 * i + 32]))
            n = len(want[0])
            assert np.array_equal(byte[:n], want[1]), i
            assert np.array_equal(codes[:n], want[0]), (i, np.argwhere(codes[:n] != want[0])[:4])
    k, v = kept_values(cfg, packed, 0, 0, len(rows))
    assert np.array_equal(f64(back.k_ret[0, 0]), k) and np.array_equal(f64(back.v_ret[0, 0]), v)
