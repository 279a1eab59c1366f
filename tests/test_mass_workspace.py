"""Room that the weights of a prompt ask for (CPU: the size query and the check of a call, nothing is launched)."""
import pytest

from paper_2510_20787_amd import binding as B
from tests.test_kept_abi import EINVAL, EWORKSPACE, P, mass


@pytest.mark.parametrize("dtype,Hkv,D", [("bf16", 8, 64), ("bf16", 32, 128), ("f32", 2, 64)])
@pytest.mark.parametrize("window", [1, 2048, 1 << 20, (1 << 31) - 1])
def test_room_grows_with_the_prompt_not_with_its_square(dtype, Hkv, D, window):
    cfg = B.make_cfg(Hkv, Hkv, D, window, 0, dtype=dtype)
    for total in (1 << 15, 1 << 17, 1 << 20, 1 << 24):
        for n in (1, 7):
            most = B.ltea_mass_workspace_bytes(cfg, n, total, total)
            # 16 sums of a token, and 2048 workgroups of at most 256 keys
            assert most <= 4 * (16 * Hkv * total + 2048 * 256) + 256
            for last in (0, 1, 300, 1 << 16):
                args = dict(cfg=cfg, q_st=Hkv * D, q_sh=D, k_st=Hkv * D, k_sh=D, n=n, total=total, longest=total, last=last)
                assert mass(**args, ws=P + 16, nbytes=most) == EINVAL                       # (enough: refused for its alignment)
    # a short window: the parts that reach a key are few, however long the prompt
    cfg = B.make_cfg(Hkv, Hkv, D, 1000, 0, dtype=dtype)
    args = dict(cfg=cfg, q_st=Hkv * D, q_sh=D, k_st=Hkv * D, k_sh=D, n=1, total=1 << 20, longest=1 << 20)
    assert mass(**args, ws=P + 16, nbytes=4 * 3 * Hkv << 20) == EINVAL and mass(**args, ws=P + 16, nbytes=4 * Hkv << 20) == EWORKSPACE
