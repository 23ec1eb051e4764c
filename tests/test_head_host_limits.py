"""What the head operators refuse at the ends of their arguments' ranges, without a GPU."""
import pytest

from test_head_host import ARGS, BWD, E_VALUE, LOSS, backward, desc, lib, logits, loss  # noqa: F401

ALONE = dict(ce_grad_scale=0.0)   # CE belongs to tau = 1


@pytest.mark.parametrize("bad", [
    dict(softcap=1e-39),                     # 1 / softcap is beyond fp32
    dict(tau=1e-39, **ALONE),                # log2(e) / tau
    dict(softcap=3e38),                      # softcap log2(e)
    dict(softcap=1e30, tau=1e-10, **ALONE),  # softcap log2(e) / tau
    dict(softcap=1e-30, tau=1e30, **ALONE),  # and nothing of it
    dict(grad_scale=10.0, tau=1e-38, **ALONE),
    dict(grad_scale=3e38, ce_grad_scale=3e38),
])
def test_the_loss_refuses_scales_beyond_fp32(lib, bad):  # noqa: F811
    d = desc(**bad)
    assert lib.npd_head_workspace_bytes(d, LOSS) == 0
    if d.tau != 1.0:
        assert loss(lib, d, 1 << 25, nll=None, lse=None) == E_VALUE
    assert loss(lib, d, 1 << 25) == E_VALUE


def test_the_ends_of_the_ranges_are_taken(lib):  # noqa: F811
    for ok in (dict(softcap=2.0 ** -126), dict(softcap=2e38), dict(tau=3e38, **ALONE), dict(tau=1e-38, **ALONE),
               dict(grad_scale=3e38)):
        d = desc(**ok)
        assert lib.npd_head_workspace_bytes(d, LOSS) > 0
    # without a gradient a scale is not looked at beyond being finite
    assert lib.npd_head_workspace_bytes(desc(grad_scale=10.0, tau=1e-38, flags=0, **ALONE), LOSS) > 0


def test_logits_refuse_a_soft_cap_without_an_inverse(lib):  # noqa: F811
    assert logits(lib, desc(flags=0, softcap=1e-39)) == E_VALUE
    assert backward(lib, desc(softcap=1e-39), 1 << 25, logits=ARGS["logits"]) == E_VALUE
    # tau and the scales are the loss's
    assert lib.npd_head_workspace_bytes(desc(tau=0.0, grad_scale=float("nan")), BWD) > 0
