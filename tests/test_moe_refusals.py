"""What the operators behind the gather refuse, before anything reaches a GPU (no kernel is launched here)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2609_04609_b200 import ciera

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20  # an address that no call may follow
lib = ciera._lib


def _config(**kw):
    base = dict(n_experts=64, top_k=8, n_groups=8, top_groups=4, group_best=2, score=0, renormalise=0, scale=1.0)
    return ciera.RouteConfig(**{**base, **kw})


@pytest.mark.parametrize("bad", [
    dict(n_experts=0), dict(n_experts=1025), dict(top_k=0), dict(top_k=33), dict(top_k=33, n_experts=640), dict(n_groups=0),
    dict(n_groups=7), dict(n_groups=64), dict(top_groups=0), dict(top_groups=9), dict(group_best=0), dict(group_best=3), dict(score=2),
    dict(score=-1), dict(renormalise=2), dict(scale=float("nan")), dict(scale=float("inf")), dict(top_k=9, top_groups=1),
])
def test_route_refuses_configurations(bad):
    cfg = _config(**bad)
    assert lib.ciera_route(cfg, 0, A, 4, 1024, None, A, A, None) == ciera.ERR_INVALID_ARG
    assert lib.ciera_route_backward(cfg, 0, A, 4, 1024, A, A, A, 1024, None) == ciera.ERR_INVALID_ARG


def test_route_refuses_arguments():
    cfg = _config()
    inv, mis = ciera.ERR_INVALID_ARG, ciera.ERR_MISALIGNED
    assert lib.ciera_route(None, 0, A, 4, 64, None, A, A, None) == inv
    assert lib.ciera_route(cfg, 3, A, 4, 64, None, A, A, None) == inv
    assert lib.ciera_route(cfg, 0, None, 4, 64, None, A, A, None) == inv
    assert lib.ciera_route(cfg, 0, A, 4, 64, None, None, A, None) == inv
    assert lib.ciera_route(cfg, 0, A, 4, 64, None, A, None, None) == inv
    assert lib.ciera_route(cfg, 0, A, 4, 63, None, A, A, None) == inv
    assert lib.ciera_route(cfg, 0, A, 1 << 40, 64, None, A, A, None) == inv
    assert lib.ciera_route(cfg, 0, A + 1, 4, 64, None, A, A, None) == mis
    assert lib.ciera_route(cfg, 1, A + 2, 4, 64, None, A, A, None) == mis
    assert lib.ciera_route(cfg, 0, A, 4, 64, A + 2, A, A, None) == mis
    assert lib.ciera_route(cfg, 0, A, 4, 64, None, A + 2, A, None) == mis
    assert lib.ciera_route(cfg, 0, None, 0, 64, None, None, None, None) == ciera.OK  # no tokens
    assert lib.ciera_route_backward(cfg, 0, A, 4, 64, A, A, None, 64, None) == inv
    assert lib.ciera_route_backward(cfg, 0, A, 4, 64, A, A, A, 63, None) == inv
    assert lib.ciera_route_backward(cfg, 0, A, 4, 64, A, A, A + 1, 64, None) == mis
    assert lib.ciera_route_backward(cfg, 0, None, 0, 64, None, None, None, 64, None) == ciera.OK


def test_layout_refuses():
    inv = ciera.ERR_INVALID_ARG
    ok = [A, 100, 64, A, A, A, A, A, None]
    for i, v in ((0, None), (1, (1 << 30) + 1), (2, 0), (2, 1025), (3, None), (4, None), (5, None), (6, None), (7, None)):
        args = list(ok)
        args[i] = v
        assert lib.ciera_expert_layout(*args) == inv, i
    for i in (0, 3, 4, 5, 6, 7):
        args = list(ok)
        args[i] = A + 2
        assert lib.ciera_expert_layout(*args) == ciera.ERR_MISALIGNED, i
    assert ciera.expert_rows_capacity(0, 64) == 0 and ciera.expert_rows_capacity(1, 64) == 128
    assert ciera.expert_layout_workspace_bytes(10, 64) > 0


def _rows(**kw):
    base = dict(source=0, dtype=0, rows=256, cols=256, x_rows=256, x=A, x_stride=256, grad=None, grad_stride=0, slot_of_row=None,
                row_weights=None, starts=None, top_k=1, n_experts=0, q=A, q_stride=256, scales=A, scales_stride=256, qt=A,
                qt_stride=256, scales_t=A, scales_t_stride=256)
    return ciera._Fp8Rows(**{**base, **kw})


@pytest.mark.parametrize("bad,status", [
    (dict(source=3), -1), (dict(dtype=3), -1), (dict(cols=0), -1), (dict(rows=1 << 31), -1), (dict(x=None), -1), (dict(q=None), -1),
    (dict(scales=None), -1), (dict(qt=None), -1), (dict(scales_t=None), -1), (dict(x_stride=255), -1), (dict(q_stride=240), -1),
    (dict(scales_stride=255), -1), (dict(qt_stride=240), -1), (dict(scales_t_stride=255), -1), (dict(x_rows=255), -1),
    (dict(grad=A, grad_stride=256), -1), (dict(row_weights=A), -1), (dict(slot_of_row=A, top_k=0), -1), (dict(slot_of_row=A, top_k=33), -1),
    (dict(starts=A, n_experts=0), -1), (dict(starts=A, n_experts=1025), -1), (dict(source=1), -1), (dict(source=2, grad_stride=128), -1),
    (dict(source=2, grad=A, grad_stride=127), -1), (dict(source=2, cols=255, grad=A, grad_stride=128), -1),
    (dict(source=1, x_stride=512, slot_of_row=A, row_weights=A), -1),
    (dict(q=A + 8), -3), (dict(q_stride=264), -3), (dict(qt=A + 8), -3), (dict(qt_stride=264), -3), (dict(x=A + 1), -3),
    (dict(slot_of_row=A + 2), -3), (dict(starts=A + 1, n_experts=4), -3),
])
def test_quantize_rows_refuses(bad, status):
    assert lib.ciera_fp8_quantize_rows(_rows(**bad), None) == status


def test_quantize_of_nothing_is_nothing():
    assert lib.ciera_fp8_quantize_rows(_rows(rows=0), None) == ciera.OK
    assert lib.ciera_fp8_quantize_rows(None, None) == ciera.ERR_INVALID_ARG
    assert lib.ciera_fp8_quantize_blocks(None, None) == ciera.ERR_INVALID_ARG
    assert lib.ciera_fp8_quantize_blocks(ciera._Fp8Blocks(dtype=0, matrices=0), None) == ciera.OK


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=9), -1), (dict(rows=0), -1), (dict(cols=0), -1), (dict(x=None), -1), (dict(q=None), -1), (dict(scales=None), -1),
    (dict(qt=None), -1), (dict(x_stride=200), -1), (dict(q_stride=240), -1), (dict(scales_stride=1), -1), (dict(qt_stride=240), -1),
    (dict(scales_t_stride=1), -1), (dict(q=A + 8), -3), (dict(q_stride=264), -3), (dict(q_matrix_stride=65528), -3),
    (dict(qt_matrix_stride=65528), -3), (dict(x=A + 1), -3),
])
def test_quantize_blocks_refuses(bad, status):
    base = dict(dtype=0, matrices=2, rows=256, cols=256, x=A, x_stride=256, x_matrix_stride=65536, q=A, q_stride=256, q_matrix_stride=65536,
                scales=A, scales_stride=2, scales_matrix_stride=4, qt=A, qt_stride=256, qt_matrix_stride=65536, scales_t=A,
                scales_t_stride=2, scales_t_matrix_stride=4)
    assert lib.ciera_fp8_quantize_blocks(ciera._Fp8Blocks(**{**base, **bad}), None) == status


@pytest.mark.parametrize("bad,status", [
    (dict(mode=3), -1), (dict(out_dtype=4), -1), (dict(m=0), -1), (dict(n=0), -1), (dict(k=0), -1), (dict(m=1 << 31), -1), (dict(a=None), -1),
    (dict(a_scales=None), -1), (dict(b=None), -1), (dict(b_scales=None), -1), (dict(out=None), -1), (dict(b_blocks=2), -1),
    (dict(mode=1), -1), (dict(mode=1, b_blocks=1, b_scales_stride=2), -1), (dict(mode=2), -1), (dict(mode=2, starts=A, n_experts=0), -1),
    (dict(mode=2, starts=A, n_experts=4, b_blocks=1), -1), (dict(starts=A), -1), (dict(mode=1, starts=A, n_experts=1025, b_blocks=1), -1),
    (dict(a_stride=240), -1), (dict(b_stride=240), -1), (dict(a_scales_stride=255), -1), (dict(b_scales_stride=255), -1),
    (dict(b_blocks=1, b_scales_stride=1), -1), (dict(out_stride=255), -1),
    (dict(a=A + 8), -3), (dict(b=A + 8), -3), (dict(a_stride=264), -3), (dict(b_stride=264), -3), (dict(out=A + 2), -3),
    (dict(mode=1, starts=A, n_experts=4, b_blocks=1, b_scales_stride=2, b_matrix_stride=65528), -3), (dict(status=A + 2), -3),
    (dict(a_stride=1 << 40), -2), (dict(b_stride=1 << 40), -2),
])
def test_matmul_refuses(bad, status):
    base = dict(mode=0, out_dtype=1, b_blocks=0, n_experts=0, m=256, n=256, k=256, a=A, a_stride=256, a_scales=A, a_scales_stride=256, b=A,
                b_stride=256, b_matrix_stride=65536, b_scales=A, b_scales_stride=256, b_scales_matrix_stride=4, starts=None, out=A,
                out_stride=256, out_matrix_stride=65536, status=None)
    assert lib.ciera_fp8_matmul(ciera._Fp8Product(**{**base, **bad}), None) == status


def test_combine_refuses():
    ok = [0, A, 512, 256, A, A, 64, 8, 256, A, 256, None]
    for i, v, status in ((0, 5, -1), (1, None, -1), (2, 1 << 31, -1), (3, 255, -1), (4, None, -1), (6, 1 << 31, -1), (7, 0, -1), (7, 33, -1),
                         (8, 0, -1), (9, None, -1), (10, 255, -1), (1, A + 1, -3), (4, A + 2, -3), (5, A + 2, -3), (9, A + 1, -3)):
        args = list(ok)
        args[i] = v
        assert lib.ciera_expert_combine(*args) == status, (i, v)
    assert lib.ciera_expert_combine(0, A, 512, 256, None, None, 0, 8, 256, None, 256, None) == ciera.OK
    back = [0, A, 256, A, 512, 256, A, A, 64, 8, 256, A, A, 256, None]
    for i, v, status in ((1, None, -1), (2, 255, -1), (3, None, -1), (6, None, -1), (11, None, -1), (13, 255, -1), (11, A + 2, -3), (12, A + 1, -3)):
        args = list(back)
        args[i] = v
        assert lib.ciera_expert_combine_backward(*args) == status, (i, v)


def _refused(f, *args, **kw):
    with pytest.raises(ciera.CieraError) as e:
        f(*args, **kw)
    assert e.value.status in (ciera.ERR_INVALID_ARG, ciera.ERR_CAPACITY)


def test_binding_refuses_what_is_not_on_a_gpu_or_not_a_tensor():
    cfg = _config()
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    i, w = torch.zeros(4, 8, dtype=torch.int32), torch.zeros(4, 8)
    q = torch.zeros(4, 64, dtype=torch.float8_e4m3fn)
    s = torch.zeros(1, 16, dtype=torch.uint8)
    for bad in (x, None, np.zeros((4, 64)), 7):
        _refused(ciera.route, cfg, bad, None, i, w)
        _refused(ciera.route_backward, cfg, bad, i, w, x)
        _refused(ciera.expert_layout, bad, 64, i, i, i, i, i)
        _refused(ciera.fp8_quantize_rows, bad, q, s)
        _refused(ciera.fp8_quantize_blocks, bad, q, s)
        _refused(ciera.fp8_matmul, bad, s, q, s, x)
        _refused(ciera.expert_combine, bad, i, w, x)
        _refused(ciera.expert_combine_backward, x, bad, i, w, w)


def test_structures_are_laid_out_as_in_the_header(tmp_path):
    structs = {"ciera_fp8_rows": ciera._Fp8Rows, "ciera_fp8_blocks": ciera._Fp8Blocks, "ciera_fp8_product": ciera._Fp8Product,
               "ciera_route_config": ciera.RouteConfig}
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "ciera.h"', "int main(void) {"]
    for name, struct in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in struct._fields_]
    (tmp_path / "layout.c").write_text("\n".join(lines + ["return 0;", "}"]))
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", exe, str(tmp_path / "layout.c")], check=True)
    said = dict(line.split() for line in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines())
    for name, struct in structs.items():
        assert int(said[name]) == ctypes.sizeof(struct), name
        for f in struct._fields_:
            assert int(said[f"{name}.{f[0]}"]) == getattr(struct, f[0]).offset, (name, f[0])


@pytest.mark.gpu
def test_binding_refuses_shapes_and_types():
    dev = "cuda:0"
    z = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device=dev)  # noqa: E731
    i32, u8, f8 = torch.int32, torch.uint8, torch.float8_e4m3fn
    cfg = _config()
    x, i, w = z(4, 64, dtype=torch.bfloat16), z(4, 8, dtype=i32), z(4, 8)
    ciera.route(cfg, x, None, i, w)
    for args in ((x[:, :63], None, i, w), (x.t(), None, i, w), (x, z(63), i, w), (x, None, i.long(), w), (x, None, i, w.half()),
                 (x, None, i[:3], w), (x, None, i, w.cpu()), (x.to(torch.int32), None, i, w), (x, None, None, w)):
        _refused(ciera.route, cfg, *args)
    _refused(ciera.route_backward, cfg, x, i, w, x.float())
    _refused(ciera.route_backward, cfg, x, i, w, x[:3])
    cap = ciera.expert_rows_capacity(32, 64)
    ok = [i, 64, z(65, dtype=i32), z(64, dtype=i32), z(4, 8, dtype=i32), z(cap, dtype=i32), z(64, dtype=u8)]
    ciera.expert_layout(*ok)
    for at, v in ((2, z(64, dtype=i32)), (3, z(63, dtype=i32)), (4, z(32, dtype=i32)), (5, z(cap - 1, dtype=i32)), (6, z(0, dtype=u8)),
                  (6, None), (0, i.long())):
        args = list(ok)
        args[at] = v
        _refused(ciera.expert_layout, *args)
    y, q, s, qt, st = z(130, 256), z(130, 256, dtype=f8), z(2, 144, dtype=u8), z(256, 144, dtype=f8)[:, :130], z(2, 256, dtype=u8)
    ciera.fp8_quantize_rows(y, q, s, qt, st)
    for args, kw in (((y, q[:, :128], s), {}), ((y, q, s[:1]), {}), ((y, q, s[:, :128]), {}), ((y, q, s, qt), {}), ((y, q, s, qt[:200], st), {}),
                     ((y, q, s, qt, st[:, :200]), {}), ((y, q, s), dict(kind=ciera.SOURCE_SWIGLU)),
                     ((y, q, s), dict(kind=ciera.SOURCE_SWIGLU_BACKWARD)), ((y, q, s), dict(grad=y)), ((y, q.view(u8), s), {}),
                     ((y, q, s), dict(slot_of_row=z(100, dtype=i32))), ((y, q, s), dict(row_weights=z(130, 1))), ((y.double(), q, s), {})):
        _refused(ciera.fp8_quantize_rows, *args, **kw)
    m = z(2, 130, 256)
    qb, sb = z(2, 130, 256, dtype=f8), z(2, 2, 2, dtype=u8)
    ciera.fp8_quantize_blocks(m, qb, sb)
    for args in ((m[0], qb, sb), (m, qb[:1], sb), (m, qb, sb[:, :1]), (m, qb, sb, z(2, 256, 144, dtype=f8)[:, :, :130])):
        _refused(ciera.fp8_quantize_blocks, *args)
    starts = torch.tensor([0, 128, 128], dtype=i32, device=dev)
    out = z(130, 130)
    ciera.fp8_matmul(q, s, q, s, out)
    ciera.fp8_matmul(q, s, qb, sb, out, starts)
    for args, kw in (((q, s, q[:, :128], s, out), {}), ((q, s, q, s, out[:, :100]), {}), ((q, s, qb, sb, out), {}), ((q, s, q, s, out, starts), {}),
                     ((q, s, qb, sb, out, starts), dict(contract=True)), ((q, s, q, s, out), dict(contract=True)),
                     ((q, s, qb[:1], sb[:1], out, starts), {}), ((q, s, q, s, out.double()), {}), ((q, s, q, s, out), dict(status=z(2, dtype=i32))),
                     ((q, s[:1], q, s, out), {}), ((q, s, q, s[:, :100], out), {})):
        _refused(ciera.fp8_matmul, *args, **kw)
    at = z(5, 2, dtype=i32)
    ciera.expert_combine(out, at, None, z(5, 130))
    for args in ((out, at, None, z(4, 130)), (out, at, None, z(5, 129)), (out, at[:, 0], None, z(5, 130)), (out, at, z(5, 3), z(5, 130)),
                 (out, at, None, z(5, 130).half())):
        _refused(ciera.expert_combine, *args)
    _refused(ciera.expert_combine_backward, z(5, 130), out, at, None, z(5, 3))
    _refused(ciera.expert_combine_backward, z(5, 130), out, at, None, z(5, 2), out[:3])
    torch.cuda.synchronize()
