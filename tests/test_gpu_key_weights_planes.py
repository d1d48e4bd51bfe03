"""Weights before and after in buffers of different lengths: refused where planes would lie apart differently, taken where there is
one plane only."""
import pytest
import torch

from gpu_helpers import note
from paper_2602_04361_amd import sparvar as sv

pytestmark = pytest.mark.gpu


def test_one_plane():
    note("[key weights] one plane")
    q, k = torch.randn(1, 2, 3, 64, device="cuda"), torch.randn(1, 1, 90, 64, device="cuda")
    lse, old = torch.full((1, 2, 3), 4.0, device="cuda"), torch.rand(1, 1, 90, device="cuda")
    want, got = torch.empty(1, 1, 90, device="cuda"), torch.full((1, 1, 200), 7.0, device="cuda")
    sv.sparvar_key_weights(q, 90, lse, want, w_old=old, k_cache=k)
    sv.sparvar_key_weights(q, 90, lse, got, w_old=old, k_cache=k)
    torch.cuda.synchronize()
    assert torch.equal(got[:, :, :90], want) and (got[:, :, 90:] == 7).all()
    with pytest.raises(sv.SparvarError, match="plane stride"):
        sv.sparvar_key_weights(q, 90, lse, torch.empty(1, 2, 200, device="cuda"), w_old=torch.rand(1, 2, 90, device="cuda"),
                               k_cache=k.expand(1, 2, 90, 64).contiguous())
