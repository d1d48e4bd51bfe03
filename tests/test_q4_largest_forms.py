"""Dense attention over the largest planes that a 4-bit cache's checks allow (2^31 codes), by every form that takes them: the
wide forms find K, V and scales by 32-bit offsets of their own."""
import pytest
import torch

from gpu_helpers import note, scale_of
from paper_2602_04361_amd import sparvar as sv
from q4_helpers import check_rows, values_of

# rows, with a workspace, the form (waves, sets, more than one part) that they take of one plane of 2^31 / d - 1 tokens
FORMS = [(1, True, (0, 0, True)), (1, False, (0, 0, False)), (100, True, (0, 1, True)), (240, True, (4, 1, True)), (500, True, (8, 1, True)),
         (4200, False, (0, 1, False)), (8200, False, (2, 4, False)), (16400, False, (4, 2, False))]


@pytest.mark.parametrize("d", [64, 128])
def test_forms(d):
    for nq, ws, form in FORMS:
        waves, sets, parts = sv.sparvar_dense_attn_q4_form(1, 1, 1, nq, 2 ** 31 // d - 1, d, ws)
        assert (waves, sets, parts > 1) == form, nq


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_largest_cache(d):
    """The weight lies on the last 64 tokens: their scores are some sqrt(d) 4, those of the first 64 a quarter of it, all others
    zero, and 2^25 e^-32 = 4e-7 of a row's sum at most is far below what check_rows allows."""
    n = 2 ** 31 // d - 1
    note(f"[largest] d={d} n={n}")
    g = torch.Generator(device="cuda").manual_seed(d)
    q4 = sv.Q4Cache.empty(1, 1, n, d)
    x = torch.zeros(2, 1, 1, n, d, dtype=torch.bfloat16, device="cuda")
    u = torch.randn(d, generator=g, device="cuda").sign()
    x[0, 0, 0, -64:] = (u * 4).bfloat16()
    x[1, 0, 0, -64:] = torch.randn(64, d, generator=g, device="cuda").bfloat16()
    x[:, 0, 0, :64] = x[:, 0, 0, -64:].flip(1) * 0.25
    sv.sparvar_kv_quantize_q4(x[0], x[1], 0, q4)
    small = sv.Q4Cache.empty(1, 1, 64, d)
    sv.sparvar_kv_quantize_q4(x[0][:, :, -64:], x[1][:, :, -64:], 0, small)
    torch.cuda.synchronize()
    k, v = values_of(small)
    del x
    torch.cuda.empty_cache()
    for nq, ws, form in FORMS:
        note(f"[largest] d={d} {nq} rows, form {form}")
        waves, sets, parts = sv.sparvar_dense_attn_q4_form(1, 1, 1, nq, n, d, ws)
        assert (waves, sets, parts > 1) == form
        q = (u * (1 + torch.arange(nq, device="cuda") % 3)[:, None] * 1.0).bfloat16()[None, None]
        size = sv.sparvar_dense_attn_q4_workspace(1, 1, 1, nq, n, d)
        work = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda") if ws else None
        o, lse = torch.empty_like(q), torch.empty(1, 1, nq, device="cuda")
        sv.sparvar_dense_attn_q4_fwd(q, q4, n, o, lse=lse, workspace=work)
        torch.cuda.synchronize()
        check_rows(o[0, 0].double().cpu().numpy(), lse[0, 0].double().cpu().numpy(), q[0, 0].double().cpu().numpy(), k[0, 0], v[0, 0],
                   scale_of(d), what=f"{nq} rows, form {form}")
    del q4, small
    torch.cuda.empty_cache()
