"""Options of a layer over the 8-bit cache: those it has reach the calls, the others of a bf16 layer are refused (host only:
the buffers are made on the CPU and nothing is called)."""
import pytest
import torch

from paper_2602_04361_amd import sparvar as sv
from paper_2602_04361_amd.pipeline import Q8SparsePath

ARGS = (sv.Geometry([1, 2, 4, 8], [1, 2, 4, 8], 4, 1), 3, [4], 1, 2, 64, 2, 1)


@pytest.mark.parametrize("option", [dict(use_schedule=True), dict(fused_decision=False), dict(local_lists=True),
                                    dict(dtype=torch.float32)])
def test_options_without_effect_are_refused(option):
    with pytest.raises(TypeError):
        Q8SparsePath(*ARGS, device="cpu", **option)


def test_options_that_apply():
    p = Q8SparsePath(*ARGS, block=32, device="cpu", prev_dilation=1, softmax_scale=0.5, projection="cover")
    assert (p.dil, p.scale, p.projection) == (1, 0.5, sv.PROJECT_COVER)
    assert p.o_S.dtype == torch.bfloat16 and all(t.dtype == torch.bfloat16 for t in p.out.values())
    # room for what the options ask
    assert p.csr[4][1].numel() == sv.sparvar_map_index_capacity(ARGS[0], 3, 4, 1, 2, 2, 1, 1, "cover")
    assert set(p.out) == {1, 2, 3, 4}
