"""Calls that would need a launch of more threads than 32 bits count are refused (CPU: nothing is launched)."""
import pytest

from paper_2510_20787_amd import binding as B
from tests.test_kept_abi import EINVAL, EUNSUPPORTED, P, mass, step


@pytest.mark.parametrize("by_mass", [True, False], ids=["mass", "packed"])
def test_steps_of_too_many_heads(by_mass):
    cfg = B.make_cfg(1, 1, 64, 1, 1)
    assert step(by_mass, cfg=cfg, n=1 << 24, ws=P + 16) == EUNSUPPORTED
    assert step(by_mass, cfg=cfg, n=(1 << 24) - 1, ws=P + 16) == EINVAL          # accepted up to the workspace's alignment
    assert step(by_mass, cfg=B.make_cfg(16, 16, 64, 1, 1), n=1 << 20, ws=P + 16) == EUNSUPPORTED


def test_weights_of_too_many_prompts():
    cfg = B.make_cfg(1, 1, 64, 4, 0)
    one = dict(cfg=cfg, q_st=64, k_st=64, longest=1, ws=P + 16)
    assert mass(n=3 << 20, total=3 << 20, **one) == EUNSUPPORTED
    assert mass(n=1 << 20, total=1 << 20, **one) == EINVAL
