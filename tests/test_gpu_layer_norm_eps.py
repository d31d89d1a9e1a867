"""An eps that a norm does not take is refused in the same way whatever its size."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [-1.0, float("nan"), float("inf"), 1e39, -1e39])
def test_refused(eps):
    from paper_2606_16907_amd import layer as L
    from paper_2606_16907_amd.tangram import TangramError
    x, w = torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda")
    for norm in (L.tg_rms_norm, L.tg_layer_norm):
        with pytest.raises(TangramError, match="eps"):
            norm(x, w, eps=eps)
