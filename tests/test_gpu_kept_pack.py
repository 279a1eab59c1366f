"""Kept rows in 4 bits and back, against the oracle's encoding (exact: the same bytes)."""
import numpy as np
import pytest
import torch

from oracle import kept_oracle as ko
from paper_2510_20787_amd import binding as B
from tests.kept_util import f64, kept_values

pytestmark = pytest.mark.gpu


def cache_of_rows(cfg, n_seqs, counts, seed):
    rng = np.random.default_rng(seed)
    cache = B.alloc_cache(cfg, n_seqs)
    for name in ("k_ret", "v_ret"):
        x = rng.standard_normal((n_seqs, cfg.Hkv, cfg.budget, cfg.D)) * np.exp(rng.uniform(-60, 60, (n_seqs, cfg.Hkv, cfg.budget, 1)))
        flat = x.reshape(-1, cfg.D)
        flat[0] = 0.0
        flat[1] = np.where(np.arange(cfg.D) % 2, -0.0, 0.0)
        flat[2, :32] = np.arange(32) * 0.25 - 4.0                      # halfway cases
        flat[3, :32] = np.linspace(-7.0, 7.0, 32)                      # at the limit of its exponent
        flat[4, :32] = np.linspace(-7.5, 7.5, 32)                      # past it
        flat[5, 3] = np.inf
        flat[6, 33] = np.nan
        flat[7] *= 1e-40 / np.abs(flat[7]).max()                       # below the smallest group
        flat[8, :32] = 3.0e38
        flat[9, :32] = 2.0 ** -120
        flat[10, :32] = 2.0 ** -121
        getattr(cache, name).copy_(torch.from_numpy(x))
    cache.ret_count.copy_(torch.tensor(counts, dtype=torch.int32)[:, None].expand(n_seqs, cfg.Hkv))
    return cache


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pack_and_unpack(D, dtype):
    cfg = B.make_cfg(4, 2, D, 16, 77, 0, 0.0, 0.0, dtype)
    counts = [77, 0, 1, 32, 45]
    cache = cache_of_rows(cfg, 5, counts, 1)
    packed = torch.full((5, 2, 3, 34 * D), 0xA5, dtype=torch.uint8, device="cuda")
    assert packed.numel() == B.ltea_packed_bytes(cfg, 5)
    B.ltea_kept_pack(cfg, cache, packed)
    back = B.alloc_cache(cfg, 5)
    back.ret_count.copy_(cache.ret_count)
    back.k_ret.fill_(3.0), back.v_ret.fill_(3.0)
    B.ltea_kept_unpack(cfg, packed, back)
    torch.cuda.synchronize()
    for b, n in enumerate(counts):
        for h in range(2):
            blocks = packed[b, h].cpu().numpy()
            for i in range(3):
                kc, vc, ke, ve = ko.read_block(blocks[i], D)
                live = max(0, min(32, n - 32 * i))
                for codes, byte, rows in ((kc, ke, cache.k_ret), (vc, ve, cache.v_ret)):
                    want = ko.encode(f64(rows[b, h, 32 * i:32 * i + live]))
                    assert np.array_equal(codes[:live], want[0]) and np.array_equal(byte[:live], want[1]), (b, h, i)
                    assert (codes[live:] == np.where(np.arange(D) % 2, 0xA, 0x5)).all() and (byte[live:] == 0xA5).all(), "slots past the count"
            k, v = kept_values(cfg, packed, b, h, n)
            for got, want in ((back.k_ret, k), (back.v_ret, v)):
                assert np.array_equal(f64(got[b, h, :n]), want, equal_nan=True)
                assert bool((got[b, h, n:] == 3.0).all())
    again = packed.clone()
    finite = back                               # packing what was unpacked gives the same bytes
    B.ltea_kept_pack(cfg, finite, again)
    assert torch.equal(again, packed)


def test_many_blocks():
    cfg = B.make_cfg(8, 8, 128, 16, 3000, 0, 0.0, 0.0, "bf16")
    rng = torch.Generator(device="cuda").manual_seed(3)
    cache = B.alloc_cache(cfg, 4)
    cache.k_ret.normal_(generator=rng), cache.v_ret.normal_(generator=rng)
    cache.ret_count.fill_(2999)
    packed = B.ltea_kept_pack(cfg, cache)
    back = B.alloc_cache(cfg, 4)
    back.ret_count.copy_(cache.ret_count)
    B.ltea_kept_unpack(cfg, packed, back)
    for x, y in ((cache.k_ret, back.k_ret), (cache.v_ret, back.v_ret)):
        g = x[:, :, :2999].float().unflatten(-1, (-1, 32))
        far = (g - y[:, :, :2999].float().unflatten(-1, (-1, 32))).abs()
        # at most half a step of 2 among the largest values, or 1 past the largest of them: a quarter of the group's largest magnitude
        assert bool((far <= g.abs().amax(-1, keepdim=True) / 4).all())
        assert bool((y[:, :, 2999:] == 0).all())
