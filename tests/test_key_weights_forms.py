"""Every form of sparvar_key_weights is run by a case that is known to take it: the library says which one (host only), so a case
that a change of the rule moves to another form fails here."""
import pytest
import torch

from gpu_helpers import note
from paper_2602_04361_amd import sparvar as sv

# keys of a workgroup (0: few queries of a key head), d, types of query: B, H, H_kv, n_q, n_kv, lengths (None: n_kv)
BF, F32 = torch.bfloat16, torch.float32
FORMS = [
    (0, 64, (BF, F32), (2, 8, 2, 24, 300, [300, 77])), (0, 128, (BF, F32), (2, 4, 2, 48, 530, None)),
    (32, 64, (BF, F32), (3, 4, 2, 70, 900, [900, 0, 33])), (32, 128, (BF, F32), (2, 2, 2, 161, 300, [31, 300])),
    (64, 64, (BF, F32), (1, 8, 8, 161, 1800, None)), (64, 128, (BF, F32), (2, 8, 8, 200, 900, [900, 65])),
    (128, 64, (BF, F32), (2, 16, 16, 161, 1000, [1000, 129])), (128, 128, (BF,), (2, 16, 16, 161, 2150, None)), (128, 128, (F32,), (1, 8, 8, 161, 2100, None)),
    (256, 64, (BF,), (1, 24, 24, 161, 1800, None)), (256, 128, (BF,), (2, 16, 16, 161, 1800, [1800, 257])),
]


def test_cases_take_their_forms():
    seen = set()
    for form, d, types, (B, H, Hkv, nq, nkv, _) in FORMS:
        for t in types:
            assert sv.sparvar_key_weights_form(B, H, Hkv, nq, nkv, d, t) == form, (d, t, B, H, nq, nkv)
            seen.add((form, d, t))
    assert seen == {(f, d, t) for d in (64, 128) for t in (BF, F32) for f in (0, 32, 64, 128, 256) if (f, t) != (256, F32)}
    # the most queries of a key head that the form of few takes
    for t, most in ((BF, 128), (F32, 96)):
        assert sv.sparvar_key_weights_form(1, 2, 1, most // 2, 50, 64, t) == 0 != sv.sparvar_key_weights_form(1, 1, 1, most + 1, 50, 64, t)


def test_refusals():
    lib = sv.load_library()
    assert lib.sparvar_key_weights_form(1, 2, 2, 1, 100, 64, sv.BF16, None) == sv.ERR_INVALID
    for bad in ((0, 2, 2, 1, 100, 64), (1, 3, 2, 1, 100, 64), (1, 2, 2, 0, 100, 64), (1, 2, 2, 1, 0, 64), (1, 2, 2, 1, 100, 96),
                (1, 2, 2, 1, 100 + (1 << 32), 64)):
        with pytest.raises(sv.SparvarError):
            sv.sparvar_key_weights_form(*bad, BF)
    with pytest.raises(sv.SparvarError):
        sv.sparvar_key_weights_form(1, 2, 2, 1, 100, 64, torch.float16)


@pytest.mark.gpu
@pytest.mark.parametrize("form,d,sizes,cache", [
    (form, d, sizes, cache) for form, d, types, sizes in FORMS for cache, t in (("bf16", BF), ("q4", BF), ("f32", F32)) if t in types])
def test_form(form, d, sizes, cache):
    """Against fp64, with weights from before, lengths of their own, queries without keys and keys past the lengths NaN."""
    from test_gpu_key_weights import run

    B, H, Hkv, nq, nkv, lens = sizes
    note(f"[key weights] form {form} {cache} d={d} {sizes}")
    assert sv.sparvar_key_weights_form(B, H, Hkv, nq, nkv, d, F32 if cache == "f32" else BF) == form
    run(cache, B, H, Hkv, nq, nkv, d, lens=lens, old=nkv // 2, decay=0.5, seed=form + d, qpad=1, empty=(0, nq - 1))
