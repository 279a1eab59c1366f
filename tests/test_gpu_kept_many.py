"""Conversions of more blocks than one launch holds."""
import pytest
import torch

from paper_2510_20787_amd import binding as B

pytestmark = pytest.mark.gpu


def test_conversions_of_very_many_heads():
    """2^24 + 77 heads of one row each (36 GB of blocks): the first, the last and those around the end of a launch as on their own."""
    cfg = B.make_cfg(1, 1, 64, 1, 1, dtype="bf16")
    n = (1 << 24) + 77
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB of free memory")
    g = torch.Generator(device="cuda").manual_seed(71)
    rows = [torch.randn((n, 1, 1, 64), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    no = torch.empty(0, dtype=torch.bfloat16, device="cuda")
    as_cache = lambda k, v: B.wrap_cache(no, no, no.float(), k, v, no.float(), no.int(), torch.ones((k.shape[0], 1), dtype=torch.int32, device="cuda"),
                                         no.int(), no.int())
    packed = B.ltea_kept_pack(cfg, as_cache(*rows))
    back = [torch.zeros_like(x) for x in rows]
    B.ltea_kept_unpack(cfg, packed, as_cache(*back))
    for part in (slice(0, 100), slice((1 << 24) - 60, n)):
        few = [x[part].contiguous() for x in rows]
        want = B.ltea_kept_pack(cfg, as_cache(*few))
        B.ltea_kept_unpack(cfg, want, as_cache(*few))
        assert torch.equal(packed[part], want)
        assert all(torch.equal(x[part], y) for x, y in zip(back, few))
        assert all(bool(x.any()) for x in few)
    assert bool((back[0].abs().amax(-1) > 0).all())
    del packed, back, rows
    torch.cuda.empty_cache()
