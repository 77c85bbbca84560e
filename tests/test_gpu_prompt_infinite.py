"""GPU: scores of all prompt queries where some keys have an infinite element.  All queries point away from it, so its logits are minus
infinity, it is paid nothing, and every other key what it would be paid without it."""
import pytest
import torch

from tests.test_gpu_operators import check_prompt, prompt_case, prompt_reference, say

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


SHAPES = [(2, 2, 64, 40), (2, 2, 128, 203), (7, 1, 64, 256), (2, 2, 128, 300), (7, 1, 64, 517), (32, 8, 128, 2020), (64, 64, 64, 1900)]


def scores(eng, q, k, lse=None):
    eng.psi.fill_(-1.0)
    eng.score_prompt(0, 1, q, k, row_lse=lse)
    torch.cuda.synchronize()
    return eng.psi.clone()


@pytest.mark.parametrize("Hq,H,d,L", SHAPES)
@pytest.mark.parametrize("what", ["query", "normaliser"])
def test_prompt_scores_behind_a_query_that_is_no_number(Hq, H, d, L, what):
    """The keys up to its own get no number from it, those behind it, which it does not see, what they get without it, bit for bit.
    Normalisers of minus infinity likewise."""
    eng, q, k = prompt_case(1, 1, Hq, H, d, L)
    lse = torch.rand(1, 1, Hq, L, generator=torch.Generator().manual_seed(L)).to(q.device) + 8.0 if what == "normaliser" else None
    good = scores(eng, q, k, lse)
    for r in sorted(r for r in {0, 1, 5, 37, 70, L // 2, L - 2, L - 1} if r < L):
        bad, bad_lse = q.clone(), None if lse is None else lse.clone()
        if lse is None:
            bad[:, :, :, r, 7] = float("nan")
        else:
            bad_lse[..., r] = float("nan") if r % 2 else -float("inf")
        say(f"{what} {r} of {Hq}/{H} d={d} L={L}")
        got = scores(eng, bad, k, bad_lse)
        assert torch.isfinite(good).all() and torch.equal(good[..., r + 1:], got[..., r + 1:])
        assert not torch.isfinite(got[..., :r + 1]).any()
    eng.close()


@pytest.mark.parametrize("Hq,H,d,L", SHAPES)
def test_prompt_scores_behind_a_query_that_sees_nothing(Hq, H, d, L):
    """The first key's logits are minus infinity, so that the first query has no weights, and the others get what they get in a prompt
    without it.  (The bound of check_prompt.)"""
    eng, q, k = prompt_case(1, 1, Hq, H, d, L)
    q[..., 5] = -0.5
    k[:, :, :, 0, 5] = float("inf")
    say(f"nothing to see, {Hq}/{H} d={d} L={L}")
    got = scores(eng, q, k)[0, 0]
    ref, _ = prompt_reference(q[0, 0, :, 1:], k[0, 0, :, 1:], Hq // H)
    assert not torch.isfinite(got[:, 0]).any()
    assert float(((got[:, 1:].double() - ref).abs() / (ref.abs() + 1e-8)).max()) < 2e-4
    eng.close()
