"""What the 4-bit operands and the layer for a few tokens refuse, before anything reaches a GPU (no kernel is launched here)."""
import pytest
import torch

from paper_2609_04609_b200 import ciera

A = 1 << 20  # an address that no call may follow
lib = ciera._lib


def _args(kind, base, bad):
    return kind(**{**base, **bad})


ROWS = dict(source=0, dtype=0, rows=256, cols=256, x_rows=256, x=A, x_stride=256, slot_of_row=None, starts=None, top_k=1, n_experts=0, q=A,
            q_stride=128, scales=A, scales_stride=1024)


@pytest.mark.parametrize("bad,status", [
    (dict(source=2), -1), (dict(source=3), -1), (dict(dtype=3), -1), (dict(cols=0), -1), (dict(rows=1 << 31), -1), (dict(x=None), -1),
    (dict(q=None), -1), (dict(scales=None), -1), (dict(x_stride=255), -1), (dict(q_stride=112), -1), (dict(scales_stride=512), -1),
    (dict(x_rows=255), -1), (dict(slot_of_row=A, top_k=0), -1), (dict(slot_of_row=A, top_k=33), -1), (dict(starts=A, n_experts=0), -1),
    (dict(starts=A, n_experts=1025), -1), (dict(source=1), -1), (dict(source=1, x_stride=512, slot_of_row=A, x_rows=100), -1),
    (dict(q=A + 8), -3), (dict(q_stride=136), -3), (dict(scales=A + 8), -3), (dict(scales_stride=1040), -3), (dict(x=A + 1), -3),
    (dict(slot_of_row=A + 2), -3), (dict(starts=A + 1, n_experts=4), -3),
])
def test_quantize_rows_refuses(bad, status):
    assert lib.ciera_fp4_quantize_rows(_args(ciera._Fp4Rows, ROWS, bad), None) == status


MATRICES = dict(dtype=0, matrices=2, rows=256, cols=256, x=A, x_stride=256, x_matrix_stride=65536, q=A, q_stride=128, q_matrix_stride=32768,
                scales=A, scales_stride=1024, scales_matrix_stride=2048, qt=A, qt_stride=128, qt_matrix_stride=32768, scales_t=A,
                scales_t_stride=1024, scales_t_matrix_stride=2048)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=9), -1), (dict(matrices=65536), -1), (dict(x=None), -1), (dict(q=None), -1), (dict(scales=None), -1), (dict(qt=None), -1),
    (dict(scales_t=None), -1), (dict(q=None, scales=None, qt=None, scales_t=None), -1), (dict(x_stride=200), -1), (dict(q_stride=112), -1),
    (dict(scales_stride=512), -1), (dict(qt_stride=112), -1), (dict(scales_t_stride=512), -1), (dict(q=A + 8), -3), (dict(q_stride=136), -3),
    (dict(q_matrix_stride=32776), -3), (dict(qt_matrix_stride=32776), -3), (dict(scales_t=A + 4), -3), (dict(scales_matrix_stride=2052), -3),
    (dict(x=A + 1), -3),
])
def test_quantize_matrices_refuses(bad, status):
    assert lib.ciera_fp4_quantize_matrices(_args(ciera._Fp4Matrices, MATRICES, bad), None) == status


VALUES = dict(dtype=0, matrices=2, rows=256, cols=256, q=A, q_stride=128, q_matrix_stride=32768, scales=A, scales_stride=1024,
              scales_matrix_stride=2048, out=A, out_stride=256, out_matrix_stride=65536)


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=9), -1), (dict(matrices=65536), -1), (dict(out=None), -1), (dict(q=None), -1), (dict(scales=None), -1), (dict(out_stride=255), -1),
    (dict(q_stride=112), -1), (dict(scales_stride=512), -1), (dict(out=A + 1), -3), (dict(q=A + 4), -3), (dict(scales_stride=1030), -3),
])
def test_values_refuses(bad, status):
    assert lib.ciera_fp4_values(_args(ciera._Fp4Values, VALUES, bad), None) == status


def test_nothing_is_nothing():
    for f, kind in ((lib.ciera_fp4_quantize_rows, ciera._Fp4Rows), (lib.ciera_fp4_quantize_matrices, ciera._Fp4Matrices),
                    (lib.ciera_fp4_values, ciera._Fp4Values)):
        assert f(None, None) == ciera.ERR_INVALID_ARG
    assert lib.ciera_fp4_quantize_rows(_args(ciera._Fp4Rows, ROWS, dict(rows=0)), None) == ciera.OK
    assert lib.ciera_fp4_quantize_matrices(_args(ciera._Fp4Matrices, MATRICES, dict(matrices=0)), None) == ciera.OK
    assert lib.ciera_fp4_values(_args(ciera._Fp4Values, VALUES, dict(rows=0)), None) == ciera.OK
    assert lib.ciera_fp4_matmul(None, None) == ciera.ERR_INVALID_ARG
    assert lib.ciera_expert_tokens(None, None) == ciera.ERR_INVALID_ARG


PRODUCT = dict(mode=1, out_dtype=0, n_experts=4, m=512, n=256, k=256, a=A, a_stride=128, a_scales=A, a_scales_stride=1024, b=A, b_stride=128,
               b_matrix_stride=32768, b_scales=A, b_scales_stride=1024, b_scales_matrix_stride=2048, starts=A, out=A, out_stride=256, status=A)


@pytest.mark.parametrize("bad,status", [
    (dict(mode=2), -1), (dict(mode=3), -1), (dict(out_dtype=3), -1), (dict(m=0), -1), (dict(n=0), -1), (dict(k=0), -1), (dict(m=1 << 31), -1),
    (dict(a=None), -1), (dict(a_scales=None), -1), (dict(b=None), -1), (dict(b_scales=None), -1), (dict(out=None), -1), (dict(starts=None), -1),
    (dict(mode=0), -1), (dict(n_experts=0), -1), (dict(n_experts=1025), -1), (dict(a_stride=112), -1), (dict(b_stride=112), -1),
    (dict(a_scales_stride=512), -1), (dict(b_scales_stride=512), -1), (dict(out_stride=255), -1), (dict(a=A + 8), -3), (dict(b=A + 8), -3),
    (dict(a_stride=136), -3), (dict(b_stride=136), -3), (dict(b_matrix_stride=32776), -3), (dict(a_scales=A + 8), -3),
    (dict(b_scales_stride=1040), -3), (dict(b_scales_matrix_stride=2056), -3), (dict(out=A + 1), -3), (dict(starts=A + 2), -3),
    (dict(status=A + 2), -3), (dict(a_stride=1 << 40), -2), (dict(b_matrix_stride=1 << 40), -2),
])
def test_product_refuses(bad, status):
    assert lib.ciera_fp4_matmul(_args(ciera._Fp4Product, PRODUCT, bad), None) == status


def _route(**kw):
    return ciera.RouteConfig(**{**dict(n_experts=8, top_k=2, n_groups=1, top_groups=1, group_best=2, score=0, renormalise=0, scale=1.0), **kw})


TOKENS = dict(format=0, dtype=0, logits_dtype=0, n_tokens=4, d_model=256, d_ff=128, x=A, x_stride=256, logits=A, logits_stride=8, bias=None,
              w1=A, w1_stride=256, w1_matrix_stride=65536, w1_scales=A, w1_scales_stride=2, w1_scales_matrix_stride=4, w2=A, w2_stride=128,
              w2_matrix_stride=32768, w2_scales=A, w2_scales_stride=1, w2_scales_matrix_stride=2, out=A, out_stride=256, experts=A, weights=A,
              workspace=A, workspace_bytes=1 << 20)
FOUR = dict(format=1, w1_stride=128, w1_matrix_stride=32768, w1_scales_stride=1024, w1_scales_matrix_stride=2048, w2_stride=64,
            w2_matrix_stride=16384, w2_scales_stride=512, w2_scales_matrix_stride=1024)


@pytest.mark.parametrize("bad,status", [
    (dict(format=2), -1), (dict(dtype=3), -1), (dict(logits_dtype=3), -1), (dict(n_tokens=65), -1), (dict(d_model=0), -1), (dict(d_model=200), -1),
    (dict(d_ff=64), -1), (dict(d_model=65664), -1), (dict(x=None), -1), (dict(out=None), -1), (dict(w1=None), -1), (dict(w1_scales=None), -1),
    (dict(w2=None), -1), (dict(w2_scales=None), -1), (dict(workspace=None), -1), (dict(logits=None), -1), (dict(experts=None), -1),
    (dict(weights=None), -1), (dict(x_stride=255), -1), (dict(out_stride=255), -1), (dict(logits_stride=7), -1), (dict(w1_stride=240), -1),
    (dict(w1_scales_stride=1), -1), (dict(w2_stride=112), -1), (dict(route=_route(top_k=9)), -1), (dict(route=_route(n_experts=0)), -1),
    (dict(w1=A + 8), -3), (dict(w1_stride=264), -3), (dict(w1_matrix_stride=65544), -3), (dict(w2=A + 4), -3), (dict(x=A + 1), -3),
    (dict(out=A + 1), -3), (dict(workspace=A + 8), -3), (dict(bias=A + 2), -3), (dict(experts=A + 2), -3), (dict(workspace_bytes=100), -4),
    ({**FOUR, "w1_scales": A + 4}, -3), ({**FOUR, "w1_scales_stride": 1040}, -3), ({**FOUR, "w1_scales_stride": 512}, -1),
    ({**FOUR, "w2_scales_matrix_stride": 1032}, -3), ({**FOUR, "w2_stride": 48}, -1),
])
def test_tokens_refuses(bad, status):
    assert lib.ciera_expert_tokens(_args(ciera._ExpertTokens, dict(TOKENS, route=_route()), bad), None) == status


def test_no_tokens_is_nothing():
    none = {k: None for k in ("x", "logits", "w1", "w1_scales", "w2", "w2_scales", "out", "experts", "weights", "workspace")}
    args = dict(TOKENS, route=_route(), n_tokens=0, workspace_bytes=0, **none)
    assert lib.ciera_expert_tokens(ciera._ExpertTokens(**args), None) == ciera.OK


def test_binding_refuses_what_is_not_on_a_gpu_or_has_another_shape():
    x, q, s = torch.zeros(4, 64), torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(1, 1, 512, dtype=torch.uint8)
    for call in (lambda: ciera.fp4_quantize_rows(x, q, s), lambda: ciera.fp4_values(q, s, x), lambda: ciera.fp4_matmul(q, s, q, s, x),
                 lambda: ciera.fp4_quantize_matrices(x[None], q[None], s[None]),
                 lambda: ciera.expert_tokens(_route(), x, x, None, q, s, q, s, x, q, x, q)):
        with pytest.raises(ciera.CieraError):
            call()


def test_layer_in_4_bits_is_not_for_training():
    from paper_2609_04609_b200.experts import ExpertLayer

    for kw in (dict(weight_bits=4), dict(weight_bits=3, training=False)):
        with pytest.raises(ValueError):
            ExpertLayer(None, 8, 256, 128, 2, 4, **kw)
