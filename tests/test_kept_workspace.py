"""Workspace of the steps over kept entries: scores only where a step keeps them there, and nothing behind what the queries say."""
import pytest
import torch

from paper_2510_20787_amd import binding as B
from tests.test_kept_abi import EINVAL, EWORKSPACE, P, step

SHAPES = [("bf16", 32, 8, 64, 768, 2001), ("bf16", 32, 1, 128, 512, 8192), ("f32", 4, 2, 64, 100, 300), ("bf16", 256, 2, 128, 64, 70000),
          ("bf16", 512, 256, 64, 20, 64), ("bf16", 4, 4, 64, 30, 0)]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,window,budget", SHAPES)
def test_steps_by_given_keys_need_no_room_for_scores(dtype, Hq, Hkv, D, window, budget):
    cfg = B.make_cfg(Hq, Hkv, D, window, budget, dtype=dtype)
    sizes = [B.ltea_decode_packed_workspace_bytes(cfg, n) for n in (0, 1, 2, 7, 8, 32, 33, 64, 128, 129, 256, 300, 1000)]
    assert sizes == sorted(sizes) and sizes[0] == 0 and all(x % 256 == 0 for x in sizes)
    G = Hq // Hkv
    for n, most in zip((1, 8, 300), (sizes[1], sizes[4], sizes[11])):
        # a head's plan, and as many shares as heads or CUs there are
        heads = n * Hkv
        assert most <= 4 * (heads * (4 + 2 * G + D) + max(heads, 256) * (4 + G + D + G * (D + 2)) + 2 * 64) + 256
        assert most < B.ltea_decode_kept_workspace_bytes(cfg, n)
        assert step(False, cfg=cfg, n=n, ws=P + 16, nbytes=most) == EINVAL              # enough: refused for its alignment only
    assert B.ltea_decode_packed_workspace_bytes(cfg, -1) == 0


def test_scores_that_lie_in_lds_take_no_room():
    cfg = B.make_cfg(16, 16, 128, 1024, 512, dtype="bf16")
    few, many = B.ltea_decode_kept_workspace_bytes(cfg, 16), B.ltea_decode_kept_workspace_bytes(cfg, 512)
    records = lambda heads: 4 * heads * (4 + 2 + 128 + 4 + 1 + 128 + 130)
    assert few >= records(256) and many <= records(16 * 512) + 256 * 1536 * 4 + 1024
    # scores of 16896 slots do not fit LDS
    cfg = B.make_cfg(16, 16, 128, 512, 16384, dtype="bf16")
    assert B.ltea_decode_kept_workspace_bytes(cfg, 512) >= 16 * 512 * 16896 * 4
    assert step(True, cfg=cfg, n=512, ws=P, nbytes=16 * 512 * 16896 * 4 - 1) == EWORKSPACE


FORMS = [  # sequences, Hq, Hkv, D, window, budget: whole heads with scores in LDS and not, four and eight waves, shares, two launches
    (20, 8, 2, 64, 70, 100), (150, 8, 2, 64, 45, 70), (70, 2, 2, 128, 70, 100), (70, 32, 2, 64, 90, 400), (150, 32, 2, 64, 90, 400),
    (1, 8, 2, 64, 100, 2300), (1, 18, 2, 128, 100, 2300), (1, 256, 256, 64, 20, 33), (3, 4, 2, 64, 33, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(map(str, f)))
def test_steps_stay_within_their_workspace(form):
    """Both queries' bytes are all that is written, and the results are those with room to spare."""
    from tests.kept_util import clone, make_state, step_inputs
    nb, Hq, Hkv, D, window, budget = form
    cfg = B.make_cfg(Hq, Hkv, D, window, budget, 1, 0.0, 0.0, "bf16")
    first = make_state(cfg, [window + budget + 9 + i for i in range(nb)], [budget - (i % 2 if budget else 0) for i in range(nb)], 81)
    first.n_scored.copy_(first.n_seen)
    q, k, v = step_inputs(cfg, nb, 82)
    rows = B.ltea_kept_pack(cfg, first)
    for by_mass, size in ((True, B.ltea_decode_kept_workspace_bytes(cfg, nb)), (False, B.ltea_decode_packed_workspace_bytes(cfg, nb))):
        for packed in ((None, rows) if by_mass else (rows,)):
            got = []
            for room in (0, 1 << 22):
                ws = torch.full((size + room + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
                cache, pk = clone(first), None if packed is None else packed.clone()
                call = B.ltea_decode_step_mass if by_mass else B.ltea_decode_step_packed
                out = call(cfg, q, k, v, cache, pk, workspace=ws[:size + room])
                torch.cuda.synchronize()
                assert bool((ws[size:] == 0xA5).all())
                got.append((out, torch.nan_to_num(cache.win_score), torch.nan_to_num(cache.ret_score), cache.ret_pos, cache.n_seen))
            assert all(torch.equal(a, b) for a, b in zip(*got))
