"""Refusals of the 8-bit row operators: every argument is checked before anything is launched, so these calls never touch
the HIP runtime (no accepted call is made: the pointers are fake)."""
import ctypes
import os
import shutil
import subprocess

import pytest

import quant_ref as R
from paper_2601_20655_amd import binding as B

FAKE = 0x1000


def quant(M=4, N=64, ldx=None, ldq=None, x_dtype=B.DIT_BF16, act=0, flags=0, x=FAKE, q=FAKE, scale=FAKE):
    p = B.dit_quant_rows_params(M, N, N if ldx is None else ldx, N if ldq is None else ldq, x_dtype, act, flags)
    return B.lib().dit_quant_rows_forward(x, q, scale, ctypes.byref(p), None)


def norm(M=4, N=64, ldx=None, ldr=None, ldh=None, ldq=None, eps=1e-6, x_dtype=B.DIT_BF16, r_dtype=B.DIT_BF16, flags=0,
         x=FAKE, residual=FAKE, gamma=FAKE, h=FAKE, q=FAKE, scale=FAKE):
    ld = [N if v is None else v for v in (ldx, ldr, ldh, ldq)]
    p = B.dit_norm_quant_params(M, N, *ld, eps, x_dtype, r_dtype, flags)
    return B.lib().dit_rms_norm_quant_forward(x, residual, gamma, h, q, scale, ctypes.byref(p), None)


def dequant(M=4, N=64, ldq=None, ldy=None, out_dtype=B.DIT_BF16, flags=0, q=FAKE, scale=FAKE, y=FAKE):
    p = B.dit_dequant_rows_params(M, N, N if ldq is None else ldq, N if ldy is None else ldy, out_dtype, flags)
    return B.lib().dit_dequant_rows_forward(q, scale, y, ctypes.byref(p), None)


def linear(M=4, N=64, K=64, ldx=None, ldw=None, ldy=None, out_dtype=B.DIT_BF16, flags=0, x=FAKE, xs=FAKE, w=FAKE, ws=FAKE,
           bias=None, y=FAKE):
    p = B.dit_linear_params(M, N, K, K if ldx is None else ldx, K if ldw is None else ldw, N if ldy is None else ldy,
                            out_dtype, flags)
    return B.lib().dit_linear_quant_forward(x, xs, w, ws, bias, y, ctypes.byref(p), None)


INVALID, UNSUPPORTED, ALIGNMENT = B.DIT_ERR_INVALID_ARG, B.DIT_ERR_UNSUPPORTED, B.DIT_ERR_ALIGNMENT


@pytest.mark.parametrize("call,kw,want", [
    *[(quant, kw, INVALID) for kw in (dict(x=None), dict(q=None), dict(scale=None), dict(M=0), dict(N=0), dict(M=-1),
                                      dict(ldx=56), dict(ldq=48), dict(x_dtype=2), dict(act=2), dict(act=-1), dict(flags=1))],
    (quant, dict(N=65537, ldx=65544, ldq=65552), UNSUPPORTED),
    *[(quant, kw, ALIGNMENT) for kw in (dict(x=FAKE + 8), dict(q=FAKE + 8), dict(scale=FAKE + 2), dict(ldx=68), dict(ldq=72),
                                        dict(x_dtype=B.DIT_F32, ldx=66))],
    *[(norm, kw, INVALID) for kw in (dict(x=None), dict(q=None), dict(scale=None), dict(M=0), dict(N=0), dict(ldx=56),
                                     dict(ldr=56), dict(ldh=56), dict(ldq=48), dict(x_dtype=2), dict(r_dtype=2),
                                     dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(residual=None),
                                     dict(flags=1))],
    (norm, dict(N=65537, ldx=65544, ldr=65544, ldh=65544, ldq=65552), UNSUPPORTED),
    *[(norm, kw, ALIGNMENT) for kw in (dict(x=FAKE + 8), dict(residual=FAKE + 2), dict(h=FAKE + 4), dict(gamma=FAKE + 8),
                                       dict(q=FAKE + 8), dict(scale=FAKE + 2), dict(ldx=68), dict(ldr=68), dict(ldh=68),
                                       dict(ldq=72), dict(r_dtype=B.DIT_F32, ldr=66))],
    *[(dequant, kw, INVALID) for kw in (dict(q=None), dict(scale=None), dict(y=None), dict(M=0), dict(N=0), dict(ldq=48),
                                        dict(ldy=56), dict(out_dtype=2), dict(flags=1))],
    *[(dequant, kw, ALIGNMENT) for kw in (dict(q=FAKE + 8), dict(y=FAKE + 8), dict(scale=FAKE + 1), dict(ldq=72), dict(ldy=68))],
    *[(linear, kw, INVALID) for kw in (dict(x=None), dict(xs=None), dict(w=None), dict(ws=None), dict(y=None), dict(M=0),
                                       dict(N=0), dict(K=0), dict(ldx=48), dict(ldw=48), dict(ldy=56), dict(out_dtype=2),
                                       dict(flags=1))],
    *[(linear, kw, UNSUPPORTED) for kw in (dict(K=131072), dict(ldx=(1 << 23) + 16), dict(ldw=(1 << 23) + 16))],
    *[(linear, kw, ALIGNMENT) for kw in (dict(x=FAKE + 8), dict(w=FAKE + 8), dict(y=FAKE + 8), dict(xs=FAKE + 2),
                                         dict(ws=FAKE + 4), dict(bias=FAKE + 4), dict(ldx=72), dict(ldw=72), dict(ldy=68),
                                         dict(out_dtype=B.DIT_F32, ldy=66))],
])
def test_refusals(call, kw, want):
    assert call(**kw) == want
    assert B.dit_last_hip_error() == ""


def test_null_params():
    L = B.lib()
    assert L.dit_quant_rows_forward(FAKE, FAKE, FAKE, None, None) == INVALID
    assert L.dit_rms_norm_quant_forward(FAKE, None, None, None, FAKE, FAKE, None, None) == INVALID
    assert L.dit_dequant_rows_forward(FAKE, FAKE, FAKE, None, None) == INVALID
    assert L.dit_linear_quant_forward(FAKE, FAKE, FAKE, FAKE, None, FAKE, None, None) == INVALID


def test_binding_refusals():
    """Shapes and types that the C side cannot see are refused before the library is called, on any device."""
    import torch

    x = torch.zeros((4, 64))
    q, s = torch.zeros((4, 64), dtype=torch.int8), torch.zeros(4)
    w, ws = torch.zeros((8, 64), dtype=torch.int8), torch.zeros(8)
    for f in (lambda: B.dit_quant_rows_forward(x, act="relu"),
              lambda: B.dit_quant_rows_forward(x[0]),
              lambda: B.dit_quant_rows_forward(x, q=q[:3]),
              lambda: B.dit_quant_rows_forward(x),  # not on a device
              lambda: B.dit_rms_norm_quant_forward(x, torch.ones(63)),
              lambda: B.dit_rms_norm_quant_forward(x, h_out=x),
              lambda: B.dit_rms_norm_quant_forward(x, residual=x[:3]),
              lambda: B.dit_dequant_rows_forward(q, s[:3]),
              lambda: B.dit_dequant_rows_forward(q.t(), torch.zeros(64)),
              lambda: B.dit_linear_quant_forward(q, s, w[:, :32], ws),
              lambda: B.dit_linear_quant_forward(q, s, w, s),
              lambda: B.dit_linear_quant_forward(q, s, w, ws)):
        with pytest.raises((ValueError, TypeError)):
            f()
    # a row that ends inside its last 16-byte piece, at the end of its storage
    with pytest.raises(ValueError):
        B._check_pieces("f", "x", torch.zeros(2 * 16 + 7, dtype=torch.int8).as_strided((3, 7), (16, 1)), 16)
    B._check_pieces("f", "x", torch.zeros(3 * 16, dtype=torch.int8).as_strided((3, 7), (16, 1)), 16)


@pytest.mark.parametrize("compiler,std", [("gcc", "-std=c99"), ("g++", "-std=c++17")])
def test_structs_as_c_lays_them_out(compiler, std, tmp_path):
    if shutil.which(compiler) is None:
        pytest.skip(compiler + " not found")
    structs = ["dit_quant_rows_params", "dit_norm_quant_params", "dit_dequant_rows_params", "dit_linear_params"]
    src = tmp_path / ("t.c" if compiler == "gcc" else "t.cpp")
    src.write_text('#include "dit_attn.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) {\n' + "".join(
        '  printf("%%zu %%zu\\n", sizeof(%s), offsetof(%s, flags));\n' % (s, s) for s in structs) + "  return 0;\n}\n")
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.check_call([compiler, std, "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", include, str(src), "-o", str(tmp_path / "t")])
    got = [int(x) for x in subprocess.check_output([str(tmp_path / "t")]).split()]
    assert got == [v for s in structs for v in (ctypes.sizeof(getattr(B, s)), getattr(B, s).flags.offset)]


def kernel_of(M, N, K, cus=256):
    """The kernel of a projection as quant_ref.KERNELS names it."""
    f = B.lib()._ZN3dit19choose_linear_quantEiiiiPiS0_
    f.restype = ctypes.c_int
    rows, features = ctypes.c_int(-1), ctypes.c_int(-1)
    form = f(M, N, K, cus, ctypes.byref(rows), ctypes.byref(features))
    if rows.value:
        assert form == 0 and 8 <= features.value <= 32 and rows.value in (8, 16, 32, 64)
        name = "few%d" if M <= rows.value else "blocks%d"
        assert M <= rows.value or -(-M // rows.value) * -(-N // features.value) <= cus
        return (name + "/%d") % (rows.value // 8, (features.value + 7) // 8)
    if form not in (0, 64):
        return "%d%s" % (form, " any" if K % 128 or N % 8 else "")
    return "%s%s%s" % ("64" if form else "big", " tail" if K % 128 else "", " rest" if N % 8 else "")


@pytest.mark.parametrize("kernel,M,N,K", R.KERNELS)
def test_every_kernel_has_a_shape(kernel, M, N, K):
    assert kernel_of(M, N, K) == kernel


def test_kernels_follow_rows_and_compute_units():
    """Few rows are streamed, a clip goes to 256 x 256 tiles; where a workgroup for each compute unit is not enough for the
    features, rows past 16 go to tiles; narrow outputs have no 256 x 256 form."""
    assert kernel_of(1, 15360, 5120) == "few1/4" and kernel_of(16, 5120, 20480) == "few2/3"
    assert kernel_of(17, 15360, 5120).startswith("11") and kernel_of(64, 8192, 5120) == "few8/4"
    assert kernel_of(32760, 15360, 5120) == "big" and kernel_of(32760, 15360, 5121) == "big tail"
    assert not kernel_of(1, 40960, 5120).startswith("few") and kernel_of(1, 1920, 5120, cus=32) == "few1/4"
    assert kernel_of(100000, 7, 512) .endswith(" any")
