"""CPU tests of what the layers' Python side decides about derivatives, before any launch."""
import pytest

torch = pytest.importorskip("torch")
from torch.autograd import forward_ad  # noqa: E402

from paper_2609_29119_amd import layers  # noqa: E402


@pytest.mark.parametrize("grad", [False, True])
def test_a_tangent_counts_as_training(grad):
    """Forward-mode inputs that do not require grad must not take the path without derivatives."""
    x = torch.ones(3)
    with torch.set_grad_enabled(grad):
        assert not layers._trains(x, None)
        with forward_ad.dual_level():
            d = forward_ad.make_dual(x, torch.ones(3))
            assert layers._trains(None, d) and not layers._trains(x, None)
        assert not layers._trains(d)
    assert layers._trains(x.clone().requires_grad_())
    with torch.no_grad():
        assert not layers._trains(x.clone().requires_grad_())
