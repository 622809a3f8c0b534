"""Whose advantages a policy loss is given, a sequence's or a token's: what the call says, what it leaves to their number, and what is refused (no GPU needed)."""
import pytest
import torch

from paper_2502_02406_amd import binding as B


@pytest.mark.parametrize("n,S", [(10, 4), (4, 10), (3, 3), (1, 1)])
def test_said(n, S):
    for per_token in (True, False):
        assert B._advantage_a_token("t", torch.zeros(n if per_token else S), n, S, per_token) is per_token
        if n != S:
            with pytest.raises(ValueError):
                B._advantage_a_token("t", torch.zeros(S if per_token else n), n, S, per_token)


def test_left_to_their_number():
    assert B._advantage_a_token("t", torch.zeros(4), 10, 4, None) is False
    assert B._advantage_a_token("t", torch.zeros(10), 10, 4, None) is True
    assert B._advantage_a_token("t", torch.zeros(1), 1, 1, None) is False          # (one token, one sequence: the same)
    for adv, n, S in ((3, 3, 3), (3, 10, 4), (4, 3, 3)):
        with pytest.raises(ValueError):
            B._advantage_a_token("t", torch.zeros(adv), n, S, None)


def test_types():
    for per_token in (True, False, None):
        for adv in (torch.zeros(4).double(), torch.zeros(8)[::2]):
            with pytest.raises(ValueError):
                B._advantage_a_token("t", adv, 4 if per_token else 9, 9 if per_token else 4, per_token)
