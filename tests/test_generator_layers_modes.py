"""The gated recurrence and the activations under autograd's other modes, on the host (no kernel is launched)."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2007_12792_b200 import autograd, build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def test_forward_mode_is_refused():
    """A tangent is not lost without a word: neither layer has a forward-mode derivative."""
    z, e = torch.zeros(2, 3, 4), torch.zeros(2, 4)
    with forward_ad.dual_level():
        d, de = forward_ad.make_dual(z, torch.ones_like(z)), forward_ad.make_dual(e, torch.ones_like(e))
        for call in (lambda: autograd.gated_scan(d, z), lambda: autograd.gated_scan(z, d), lambda: autograd.gated_scan(z, z, de),
                     lambda: autograd.activation(d), lambda: autograd.activation(d, "tanh", checkpoint="e4m3")):
            with pytest.raises(NotImplementedError, match="forward-mode"):
                call()
            with torch.no_grad(), pytest.raises(NotImplementedError, match="forward-mode"):
                call()
        # no tangent, or forward mode switched off: the next check of the arguments answers
        with pytest.raises(ValueError, match="CUDA"):
            autograd.gated_scan(z, z)
        with forward_ad._set_fwd_grad_enabled(False), pytest.raises(ValueError, match="CUDA"):
            autograd.activation(d)


@pytest.mark.gpu
def test_forward_mode_is_refused_on_the_device():
    z = torch.zeros(2, 3, 4, device="cuda")
    with forward_ad.dual_level():
        d = forward_ad.make_dual(z, torch.ones_like(z))
        for call in (lambda: autograd.gated_scan(d, z), lambda: autograd.gated_scan(z, d, checkpoint="int8"), lambda: autograd.activation(d)):
            with pytest.raises(NotImplementedError, match="forward-mode"):
                call()
        assert torch.equal(autograd.gated_scan(z, z)[0], z)
