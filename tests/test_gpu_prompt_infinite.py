"""GPU: scores of all prompt queries where some keys have an infinite element.  All queries point away from it, so its logits are minus
infinity, it is paid nothing, and every other key what it would be paid without it."""
import pytest
import torch

from tests.test_gpu_operators import check_prompt, prompt_case, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("NL,B,Hq,H,d,L", [(1, 1, 2, 2, 64, 203), (1, 1, 2, 2, 128, 256), (1, 1, 2, 2, 128, 257), (1, 1, 7, 1, 64, 300), (1, 1, 2, 2, 64, 320), (1, 1, 2, 2, 128, 352),
                                           (1, 1, 8, 8, 128, 1023), (1, 1, 32, 8, 128, 2020), (1, 2, 32, 32, 64, 1900), (1, 4, 32, 32, 128, 2047), (4, 4, 32, 32, 64, 1825)])
@pytest.mark.parametrize("given", [False, True])
def test_prompt_scores_of_infinite_keys(NL, B, Hq, H, d, L, given):
    """Prompts that end inside a tile of 64 rows, behind its first half and with it, in blocks of every size.  (The bound is that of
    the same scores without such keys.)"""
    eng, q, k = prompt_case(NL, B, Hq, H, d, L)
    q[..., 3] = -q[..., 3].abs() - 0.25
    at = [1, L // 2, L - 40, L - 1]
    k[..., at, 3] = float("inf")
    say(f"infinite keys {NL}x{B} {Hq}/{H} d={d} L={L} lse={given}")
    psi = check_prompt(eng, q, k, given)
    assert not psi[..., at].any() and not eng.psi[..., at].any() and torch.isfinite(eng.psi).all()
    eng.close()
