"""What the operators of a token policy refuse at the ends of their ranges, on a host without a GPU: before any HIP call."""
import ctypes as C
import re

import pytest

from paper_2509_16434_amd import learner as L

from test_token_ops_host import HP, LOSS


@pytest.mark.parametrize("scale,ent_coef", [(1e30, 1e30), (-1e25, 1e25), (3e38, 2.0)])
def test_token_loss_refuses_an_entropy_coefficient_beyond_fp32(scale, ent_coef):
    """dL/dH = -ent_coef scale weight: infinite, times entropies and probabilities of 0, it would be no number."""
    h = L.TokenHParams(**dict(HP, scale=scale, ent_coef=ent_coef))
    assert L._lib.ppo_token_loss(*dict(LOSS, hp=C.byref(h)).values()) == L.PPO_EINVAL
    assert b"product" in L._lib.ppo_last_error(None)


def test_no_form_of_the_one_launch_loss_is_built_that_no_call_reaches():
    """512 logits are 4 pieces of 16 bytes for each of 16 threads in 16 bits, 8 in 32 bits: the wider form is of 32 bits only."""
    names = set(re.findall(rb"k_token_loss_smallI(\w+?)Li(\d+)ELb[01]E", open(L.LIB_PATH, "rb").read()))
    assert {(t, k) for t, k in names} == {(b"f", b"4"), (b"f", b"8"), (b"t", b"4"), (b"DF16_", b"4")}
