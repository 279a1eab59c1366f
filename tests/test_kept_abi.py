"""Host-side checks of the calls that evict by accumulated attention weight or hold kept rows in 4 bits: every bad argument is refused
before anything could be launched (no compute call is made here)."""
import ctypes as C

import pytest
import torch

from paper_2510_20787_amd import binding as B
from tests.test_abi import good_cfg

OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, B.LTEA_EINVAL, B.LTEA_EUNSUPPORTED, B.LTEA_EWORKSPACE
P = 0x1000                                   # a pointer that is never followed
BIG = 1 << 40


def cache_at(**kw):
    fields = ("k_win", "v_win", "win_score", "k_ret", "v_ret", "ret_score", "ret_pos", "ret_count", "n_seen", "n_scored")
    return B.ltea_cache(*[kw.get(f, P) for f in fields])


def mass(cfg=None, q=P, q_st=256, q_sh=64, k=P, k_st=128, k_sh=64, cu=P, n=1, total=32, longest=32, lse=P, last=0, out=P, ws=P, nbytes=BIG):
    cfg = good_cfg() if cfg is None else cfg
    return B.lib().ltea_attention_mass(C.byref(cfg) if cfg else None, q, q_st, q_sh, k, k_st, k_sh, cu, n, total, longest, lse, last, out,
                                       ws, nbytes, None)


@pytest.mark.parametrize("case,expect", [
    (dict(cfg=False), EINVAL), (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(cu=None), EINVAL), (dict(lse=None), EINVAL),
    (dict(out=None), EINVAL), (dict(q=P + 8), EINVAL), (dict(k=P + 2), EINVAL), (dict(q_st=60), EINVAL), (dict(q_st=260), EINVAL),
    (dict(k_sh=68), EINVAL), (dict(k_st=-128), EINVAL), (dict(n=-1), EINVAL), (dict(n=0), EINVAL), (dict(total=-1), EINVAL),
    (dict(longest=31), EINVAL), (dict(longest=0), EINVAL), (dict(ws=P + 16), EINVAL), (dict(q_st=1 << 30), EUNSUPPORTED),
    (dict(total=1 << 31, longest=1 << 30, n=4), EUNSUPPORTED), (dict(total=40000, longest=40000, ws=None), EWORKSPACE),
    (dict(total=40000, longest=40000, nbytes=64), EWORKSPACE), (dict(total=0), OK), (dict(total=0, q=None, lse=None, ws=None), OK)], ids=str)
def test_mass_argument_errors(case, expect):
    assert mass(**case) == expect


def prefill(cfg=None, q=P, k=P, v=P, cu=P, n=1, total=32, longest=32, out=P, cache=None, ws=P, nbytes=BIG):
    cfg, cache = good_cfg() if cfg is None else cfg, cache_at() if cache is None else cache
    return B.lib().ltea_prefill_mass(C.byref(cfg) if cfg else None, q, 256, 64, k, v, 128, 64, cu, n, total, longest, 0, out,
                                     C.byref(cache) if cache else None, None, ws, nbytes, None)


@pytest.mark.parametrize("case,expect", [
    (dict(cfg=False), EINVAL), (dict(cache=False), EINVAL), (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL),
    (dict(cu=None), EINVAL), (dict(out=None), EINVAL), (dict(out=P + 4), EINVAL), (dict(n=-1), EINVAL), (dict(longest=3), EINVAL),
    (dict(ws=None), EWORKSPACE), (dict(nbytes=100), EWORKSPACE), (dict(ws=P + 128), EINVAL), (dict(cache=cache_at(k_win=None)), EINVAL),
    (dict(cache=cache_at(ret_score=None)), EINVAL), (dict(cache=cache_at(v_ret=P + 8)), EINVAL), (dict(cache=cache_at(n_seen=None)), EINVAL),
    (dict(n=0, total=0, longest=0), OK)], ids=str)
def test_prefill_by_mass_argument_errors(case, expect):
    assert prefill(**case) == expect


def step(by_mass, cfg=None, q=P, k=P, v=P, out=P, cache=None, packed=P, n=1, ws=P, nbytes=BIG):
    cfg, cache = good_cfg() if cfg is None else cfg, cache_at() if cache is None else cache
    head = [C.byref(cfg) if cfg else None, q, k, v, out, C.byref(cache) if cache else None, packed, n]
    if by_mass:
        return B.lib().ltea_decode_step_mass(*head, ws, nbytes, None)
    return B.lib().ltea_decode_step_packed(*head, None, ws, nbytes, None)


@pytest.mark.parametrize("by_mass", [True, False], ids=["mass", "packed"])
@pytest.mark.parametrize("case,expect", [
    (dict(cfg=False), EINVAL), (dict(cache=False), EINVAL), (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL),
    (dict(out=None), EINVAL), (dict(q=P + 8), EINVAL), (dict(out=P + 4), EINVAL), (dict(packed=P + 8), EINVAL), (dict(n=-1), EINVAL),
    (dict(n=0), OK), (dict(ws=None), EWORKSPACE), (dict(nbytes=256), EWORKSPACE), (dict(ws=P + 128), EINVAL),
    (dict(cache=cache_at(k_win=None)), EINVAL), (dict(cache=cache_at(win_score=None)), EINVAL), (dict(cache=cache_at(ret_pos=None)), EINVAL),
    (dict(cache=cache_at(ret_score=None)), EINVAL), (dict(cache=cache_at(ret_count=None)), EINVAL), (dict(cache=cache_at(n_scored=None)), EINVAL),
    (dict(cache=cache_at(v_win=P + 8)), EINVAL), (dict(packed=None, cache=cache_at(k_ret=None)), EINVAL),
    (dict(packed=None, cache=cache_at(v_ret=P + 4)), EINVAL), (dict(cfg=good_cfg(Hq=258, Hkv=2)), EUNSUPPORTED),
    # 128 heads x 2^22 slots x 4 bytes: a head's scores would pass 2^31 bytes
    (dict(cfg=good_cfg(Hq=128, Hkv=1, budget=1 << 22)), EUNSUPPORTED), (dict(n=1 << 24), EUNSUPPORTED),
    (dict(cfg=good_cfg(D=96)), EUNSUPPORTED)], ids=str)
def test_step_argument_errors(by_mass, case, expect):
    assert step(by_mass, **case) == expect


def test_step_over_packed_rows_needs_them():
    assert step(False, packed=None) == EINVAL
    # (past the check of the rows: the workspace is what is refused)
    assert step(False, packed=None, cfg=good_cfg(budget=0), cache=cache_at(k_ret=None, v_ret=None, ret_score=None, ret_pos=None), ws=None) == EWORKSPACE
    assert step(True, cache=cache_at(k_ret=None, v_ret=None), ws=None) == EWORKSPACE


@pytest.mark.parametrize("name", ["ltea_kept_pack", "ltea_kept_unpack"])
@pytest.mark.parametrize("case,expect", [
    (dict(cfg=False), EINVAL), (dict(cache=False), EINVAL), (dict(packed=None), EINVAL), (dict(packed=P + 8), EINVAL), (dict(n=-1), EINVAL),
    (dict(cache=cache_at(k_ret=None)), EINVAL), (dict(cache=cache_at(v_ret=P + 4)), EINVAL), (dict(cache=cache_at(ret_count=None)), EINVAL),
    (dict(n=1 << 30, cfg=good_cfg(budget=4096)), EUNSUPPORTED), (dict(n=0), OK), (dict(cfg=good_cfg(budget=0), packed=None), OK)], ids=str)
def test_conversion_argument_errors(name, case, expect):
    cfg, cache, packed, n = case.get("cfg", good_cfg()), case.get("cache", cache_at()), case.get("packed", P), case.get("n", 1)
    c, x = C.byref(cfg) if cfg else None, C.byref(cache) if cache else None
    args = (c, x, packed) if name == "ltea_kept_pack" else (c, packed, x)
    assert getattr(B.lib(), name)(*args, n, None) == expect


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 32, 8, 64), ("bf16", 16, 16, 128), ("f32", 2, 2, 64), ("bf16", 256, 2, 128), ("f32", 16, 1, 128)])
@pytest.mark.parametrize("window,budget", [(16, 0), (768, 512), (300, 16384), (64, 70000)])
def test_workspace_sizes_never_fall(dtype, Hq, Hkv, D, window, budget):
    cfg = B.make_cfg(Hq, Hkv, D, window, budget, dtype=dtype)
    sizes = [B.ltea_decode_kept_workspace_bytes(cfg, n) for n in (0, 1, 2, 3, 4, 7, 8, 16, 31, 32, 33, 64, 127, 128, 129, 256, 300)]
    assert sizes == sorted(sizes) and sizes[0] == 0 and all(x % 256 == 0 for x in sizes)
    for n, most in zip((1, 8, 33, 300), (sizes[1], sizes[6], sizes[10], sizes[16])):
        for packed in (P, None):             # what the size query says is enough: refused for its alignment only
            assert step(True, cfg=cfg, packed=packed, n=n, ws=P + 16, nbytes=most) == EINVAL
    for query in (B.ltea_mass_workspace_bytes, B.ltea_prefill_mass_workspace_bytes):
        by_tokens = [query(cfg, 8, t, 4096) for t in (0, 1, 100, 4096, 8000, 20000, 32768)]
        assert by_tokens == sorted(by_tokens) and by_tokens[0] == 0
        by_length = [query(cfg, 8, 8000, m) for m in (1000, 2047, 2048, 2049, 5000, 8000)]
        assert by_length == sorted(by_length)
    for total, longest in ((1, 1), (300, 300), (8000, 1000), (8000, 8000), (200000, 60000), (200000, 30000)):
        for last in (0, 1, 100, 5000):
            most = B.ltea_mass_workspace_bytes(cfg, 8, total, longest)
            assert mass(cfg, q_st=Hq * D, q_sh=D, k_st=Hkv * D, k_sh=D, n=8, total=total, longest=longest, last=last, ws=P + 16, nbytes=most) == EINVAL


def test_size_queries_of_bad_configurations_are_zero():
    bad = good_cfg(D=96)
    assert B.ltea_packed_bytes(bad, 1) == B.ltea_decode_kept_workspace_bytes(bad, 1) == B.ltea_mass_workspace_bytes(bad, 1, 1, 1) == 0
    cfg = good_cfg(budget=33)
    assert B.ltea_packed_bytes(cfg, -1) == B.ltea_decode_kept_workspace_bytes(cfg, -1) == B.ltea_mass_workspace_bytes(cfg, 1, -1, 1) == 0
    assert B.ltea_packed_bytes(cfg, 3) == 3 * cfg.Hkv * 2 * 34 * cfg.D
    assert B.ltea_decode_kept_workspace_bytes(good_cfg(Hq=258, Hkv=2), 1) == 0


def test_tensors_on_the_host_are_refused():
    """The binding refuses tensors that are not on the current device, wrong shapes and types, before the library is called."""
    cfg = good_cfg()
    cache = B.alloc_cache(cfg, 2, "cpu")
    packed = B.alloc_packed(cfg, 2, "cpu")
    assert packed.numel() == B.ltea_packed_bytes(cfg, 2)
    x = lambda h: torch.zeros(2, h, 64, dtype=torch.bfloat16)
    for call in (lambda: B.ltea_decode_step_mass(cfg, x(4), x(2), x(2), cache), lambda: B.ltea_decode_step_packed(cfg, x(4), x(2), x(2), cache, packed),
                 lambda: B.ltea_kept_pack(cfg, cache), lambda: B.ltea_kept_unpack(cfg, packed, cache),
                 lambda: B.ltea_attention_mass(cfg, x(4), x(2), torch.zeros(2, dtype=torch.int32), 2, torch.zeros(4, 2)),
                 lambda: B.ltea_prefill_mass(cfg, x(4), x(2), x(2), torch.zeros(2, dtype=torch.int32), 2, cache)):
        with pytest.raises(AssertionError):
            call()
