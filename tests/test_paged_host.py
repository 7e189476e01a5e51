"""Refusals of the paged-cache operators: every argument is checked before anything is launched, so these calls never touch the
HIP runtime (no accepted call is made: the pointers are fake); sizes of their structs."""
import ctypes
import os
import shutil
import subprocess
from types import SimpleNamespace

import pytest

from paper_2601_20655_amd import binding as B

FAKE = 0x1000
INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = (B.DIT_ERR_INVALID_ARG, B.DIT_ERR_UNSUPPORTED, B.DIT_ERR_ALIGNMENT,
                                              B.DIT_ERR_WORKSPACE)


def strides(H, D, token=None, head=None):
    return B.dit_strides(0, H * D if token is None else token, D if head is None else head)


def norm_struct(mode=0, eps=1e-6, gamma=None):
    return B.dit_qk_norm(mode, eps, gamma, gamma)


def rope(N=4, H=2, Hk=1, D=128, split=(44, 42, 42), base=1e4, in_dtype=0, out_dtype=0, flags=0, q=FAKE, k=FAKE, pos=FAKE, qo=FAKE,
         ko=FAKE, norm=None, token=None, head=None, out_token=None):
    p = B.dit_qk_rope_params(N, H, Hk, D, *split, base, in_dtype, out_dtype, flags, strides(H, D, token, head), strides(Hk, D),
                             strides(H, D, out_token), strides(Hk, D), norm or norm_struct())
    return B.lib().dit_qk_rope_forward(q, k, pos, qo, ko, ctypes.byref(p), None)


def cache_struct(n_pages=8, page_size=16, Hk=2, D=128, dtype=0, R=2, max_pages=4, page=None, token=None, head=None):
    return B.dit_kv_cache(n_pages, page_size, Hk, D, dtype, R, max_pages, page_size * Hk * D if page is None else page,
                          Hk * D if token is None else token, D if head is None else head)


def append(N=4, H=2, split=(44, 42, 42), base=1e4, in_dtype=0, out_dtype=0, flags=0, q=FAKE, k=FAKE, v=FAKE, pos=FAKE, table=FAKE,
           q_start=FAKE, kv_len=FAKE, qo=FAKE, kc=FAKE, vc=FAKE, norm=None, sk_token=None, **cache):
    c = cache_struct(**cache)
    p = B.dit_kv_append_params(N, H, *split, base, in_dtype, out_dtype, flags, strides(H, c.D), strides(c.Hk, c.D, sk_token),
                               strides(c.Hk, c.D), strides(H, c.D), norm or norm_struct(), c)
    return B.lib().dit_kv_append_forward(q, k, v, pos, table, q_start, kv_len, qo, kc, vc, ctypes.byref(p), None)


def attn_params(N=4, H=4, frame=0, window=0, max_q=0, max_kv=0, scale=0.0, q_dtype=0, out_dtype=0, flags=0, token=None, head=None,
                out_token=None, **cache):
    c = cache_struct(**cache)
    return B.dit_paged_attn_params(N, H, frame, window, max_q, max_kv, scale, q_dtype, out_dtype, flags,
                                   strides(H, c.D, token, head), strides(H, c.D, out_token), c)


def attn(q=FAKE, kc=FAKE, vc=FAKE, table=FAKE, q_start=FAKE, kv_len=FAKE, out=FAKE, lse=None, ws=FAKE, ws_bytes=1 << 40, **kw):
    p = attn_params(**kw)
    return B.lib().dit_attn_paged_forward(q, kc, vc, table, q_start, kv_len, out, lse, ctypes.byref(p), ws, ws_bytes, None)


BIG = 1 << 35  # elements of 64 GiB
CACHE_INVALID = [dict(n_pages=0), dict(page_size=0), dict(Hk=0), dict(R=0), dict(max_pages=0), dict(dtype=B.DIT_F32), dict(dtype=3),
                 dict(token=64), dict(head=64), dict(page=16 * 256 - 8), dict(token=128, head=128), dict(token=0), dict(page=-4096),
                 dict(token=-256)]
CACHE_OTHER = [(dict(D=96), UNSUPPORTED), (dict(D=256), UNSUPPORTED), (dict(page=BIG // 4), UNSUPPORTED),
               (dict(page=1 << 62), UNSUPPORTED), (dict(n_pages=2 ** 31 - 1, page=1 << 40), UNSUPPORTED)]


@pytest.mark.parametrize("call,kw,want", [
    *[(rope, kw, INVALID) for kw in (dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(N=-1), dict(H=0), dict(Hk=0),
                                     dict(q=None, qo=None), dict(q=None, qo=None, k=None, ko=None, H=0, Hk=0), dict(in_dtype=2),
                                     dict(out_dtype=3), dict(flags=1), dict(split=(44, 42, 41)), dict(split=(43, 43, 42)),
                                     dict(split=(130, -2, 0)), dict(base=0.0), dict(base=float("inf")), dict(base=float("nan")),
                                     dict(norm=norm_struct(3)), dict(norm=norm_struct(1, -1.0)),
                                     dict(norm=norm_struct(2, float("nan"))), dict(token=128), dict(head=64), dict(out_token=200))],
    *[(rope, kw, UNSUPPORTED) for kw in (dict(D=96), dict(D=256), dict(H=512, norm=norm_struct(2)),
                                         dict(H=1024, D=64, split=(22, 20, 22), norm=norm_struct(2)))],
    *[(rope, kw, ALIGNMENT) for kw in (dict(q=FAKE + 8), dict(ko=FAKE + 2), dict(pos=FAKE + 2), dict(token=260), dict(out_token=257),
                                       dict(in_dtype=1, token=258), dict(norm=norm_struct(1, 1e-6, FAKE + 8)))],
    *[(append, kw, INVALID) for kw in (dict(k=None), dict(v=None), dict(q=None), dict(qo=None), dict(table=None), dict(q_start=None),
                                       dict(kv_len=None), dict(kc=None), dict(vc=None), dict(N=-1), dict(H=0), dict(in_dtype=2),
                                       dict(out_dtype=3), dict(flags=1), dict(split=(44, 42, 40)), dict(base=-1.0),
                                       dict(norm=norm_struct(-1)), dict(sk_token=128), dict(q=None, qo=None)) + tuple(CACHE_INVALID)],
    (append, dict(H=400, Hk=64, norm=norm_struct(2)), UNSUPPORTED),
    *[(append, kw, want) for kw, want in CACHE_OTHER],
    *[(append, kw, ALIGNMENT) for kw in (dict(k=FAKE + 8), dict(v=FAKE + 4), dict(kc=FAKE + 8), dict(vc=FAKE + 8), dict(pos=FAKE + 1),
                                         dict(table=FAKE + 2), dict(q_start=FAKE + 2), dict(kv_len=FAKE + 3), dict(sk_token=260),
                                         dict(head=132, token=264, page=16 * 264), dict(page=16 * 256 + 4))],
    *[(attn, kw, INVALID) for kw in (dict(q=None), dict(kc=None), dict(vc=None), dict(table=None), dict(q_start=None),
                                     dict(kv_len=None), dict(out=None), dict(N=-1), dict(H=0), dict(H=3), dict(frame=-1),
                                     dict(window=-1, frame=1), dict(window=1), dict(max_q=-1), dict(max_kv=-1), dict(q_dtype=3),
                                     dict(out_dtype=2), dict(flags=1), dict(token=128), dict(head=8), dict(out_token=500))
      + tuple(CACHE_INVALID)],
    (attn, dict(N=2 ** 31 - 1, H=4), UNSUPPORTED),
    (attn, dict(N=1 << 27, H=8), UNSUPPORTED),
    *[(attn, kw, want) for kw, want in CACHE_OTHER],
    *[(attn, kw, ALIGNMENT) for kw in (dict(q=FAKE + 8), dict(kc=FAKE + 8), dict(vc=FAKE + 2), dict(out=FAKE + 4), dict(lse=FAKE + 2),
                                       dict(table=FAKE + 1), dict(q_start=FAKE + 2), dict(kv_len=FAKE + 2), dict(token=516),
                                       dict(out_dtype=1, out_token=514))],
    *[(attn, dict(max_pages=1000, **kw), WORKSPACE) for kw in (dict(ws=None), dict(ws=FAKE + 64), dict(ws_bytes=0))],
])
def test_rejections(call, kw, want):
    assert call(**kw) == want


def test_null_params():
    lib = B.lib()
    assert lib.dit_qk_rope_forward(FAKE, FAKE, FAKE, FAKE, FAKE, None, None) == INVALID
    assert lib.dit_kv_append_forward(*[FAKE] * 10, None, None) == INVALID
    assert lib.dit_attn_paged_forward(*[FAKE] * 8, None, FAKE, 1 << 30, None) == INVALID
    assert lib.dit_attn_paged_workspace_bytes(None) == 0


def test_no_tokens_is_no_error():
    none = dict(q=None, N=0)
    assert rope(k=None, qo=None, ko=None, **none) == B.DIT_OK
    assert append(k=None, v=None, qo=None, **none) == B.DIT_OK
    assert attn(out=None, ws=None, ws_bytes=0, **none) == B.DIT_OK


def test_workspace_size():
    """None where there are tiles enough; else as much for any counts, and short of a workspace the call is refused."""
    for kw in (dict(), dict(N=1), dict(N=300, max_pages=4000), dict(N=5000, H=40, Hk=40, max_pages=2000), dict(N=64, R=64)):
        p = attn_params(**kw)
        n = B.dit_attn_paged_workspace_bytes(p)
        assert n >= 256 and n % 256 == 0 and n < 1 << 29, kw
        if n > 256:
            assert attn(ws_bytes=n - 256, **kw) == WORKSPACE
    for bad in (dict(N=-1), dict(H=3), dict(D=96), dict(window=1)):
        assert B.dit_attn_paged_workspace_bytes(attn_params(**bad)) == 0


def plan(N, R, H, Hk, D, keys, max_q, runs=1):
    class Plan(ctypes.Structure):
        _fields_ = [("few", ctypes.c_bool), ("big", ctypes.c_bool)] + [(n, ctypes.c_int) for n in (
            "few_qb", "few_waves", "big_qb", "big_waves", "few_units", "big_units", "few_pieces", "big_pieces", "few_each", "big_each", "few_cap", "big_cap")] + [
            ("few_bytes", ctypes.c_size_t), ("big_bytes", ctypes.c_size_t)]

    f = B.lib()._ZN3dit10plan_pagedEiiiiilii
    f.restype = Plan
    f.argtypes = [ctypes.c_int] * 5 + [ctypes.c_long, ctypes.c_int, ctypes.c_int]
    return f(N, R, H, Hk, D, keys, max_q, runs)


@pytest.mark.parametrize("N,R,H,Hk,max_q,few,big", [
    (1, 1, 40, 8, 0, True, False), (32, 32, 40, 8, 1, True, False), (4680, 1, 40, 40, 4680, False, True),
    (200, 5, 6, 3, 196, True, True), (200, 5, 6, 3, 0, True, True), (2 ** 29 - 1, 2 ** 29 - 1, 1, 1, 1, True, False)])
def test_which_kernels(N, R, H, Hk, max_q, few, big):
    p = plan(N, R, H, Hk, 128, 32768, max_q)
    assert (p.few, p.big) == (few, big)
    # every call has workgroups, not more than a launch has room for
    for on, units in ((few, p.few_units), (big, p.big_units)):
        assert not on or 1 <= units <= 1 << 20


@pytest.mark.parametrize("runs", [0, 1])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Hk", [(1, 1), (8, 1), (40, 8), (40, 40)])
def test_workspace_is_bounded(H, Hk, D, runs):
    """Whatever the counts and hints: room for 2^19 rows of pieces a kernel, at most, and for every tile's pieces as planned."""
    for N in (1, 17, 500, 4680, 1_000_000):
        for requests in (1, 3, 100, 700):
            for keys in (1, 257, 8190, 100_000, 2 ** 31 - 65536):
                for max_q in (0, 1, 40, N):
                    p = plan(N, requests, H, Hk, D, keys, max_q, runs)
                    for on, size, rows, each, pieces, cap in (
                            (p.few, p.few_bytes, 16 * p.few_qb, p.few_each, p.few_pieces, p.few_cap),
                            (p.big, p.big_bytes, 16 * p.big_qb * p.big_waves, p.big_each, p.big_pieces, p.big_cap)):
                        assert size <= 2 ** 19 * (4 * D + 8) + 256 and (on or size == 0)
                        if on and each > 1:
                            assert size >= Hk * cap * rows * (4 * D + 8) and cap > pieces >= each >= 2 and each <= 512


def test_python_wrappers_check_extents_before_any_call():
    import torch

    bf = dict(dtype=torch.bfloat16)
    q, k = torch.zeros((4, 2, 128), **bf), torch.zeros((4, 1, 128), **bf)
    cache = torch.zeros((3, 16, 1, 128), **bf)
    table, starts, lens = (torch.zeros(s, dtype=torch.int32) for s in ((2, 3), (3,), (2,)))
    pos = torch.zeros((4, 3), dtype=torch.int32)
    for call in (lambda: B.dit_qk_rope_forward(q, k, pos, (44, 42, 42)), lambda: B.dit_qk_rope_forward(None, None, pos),
                 lambda: B.dit_qk_rope_forward(q[0], k, pos), lambda: B.dit_qk_rope_forward(q, k[:3], pos),
                 lambda: B.dit_kv_append_forward(k, k, cache, cache, table, starts, lens),
                 lambda: B.dit_kv_append_forward(k, k[:3], cache, cache, table, starts, lens),
                 lambda: B.dit_attn_paged_forward(q, cache, cache, table, starts, lens),
                 lambda: B.dit_attn_paged_forward(q, cache, cache, table, starts, lens, frame=(1 << 32) + 1),
                 lambda: B.dit_attn_paged_forward(q, cache, cache, table, starts, lens, frame=1, window=-1),
                 lambda: B.dit_attn_paged_forward(q, cache, cache, table, starts, lens, max_q=1 << 31),
                 lambda: B.dit_attn_paged_forward(q[0], cache, cache, table, starts, lens)):
        with pytest.raises(ValueError):
            call()


class Fake:
    """Stands for a device tensor: what the wrappers look at before they hand over pointers."""

    def __new__(cls, t, device=0):
        import torch

        class T(torch.Tensor):
            def get_device(self):
                return device

            def data_ptr(self):
                return FAKE

        return t.as_subclass(T)


def test_python_wrappers_check_shapes_types_and_devices(monkeypatch):
    """With tensors that say that they are on a device: nothing is launched, every call raises."""
    import torch

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32

    def t(shape, dtype=bf, device=0):
        return Fake(torch.zeros(shape, dtype=dtype), device)

    q, k, cache = t((4, 2, 128)), t((4, 1, 128)), t((3, 16, 1, 128))
    table, starts, lens, pos = t((2, 3), i32), t((3,), i32), t((2,), i32), t((4, 3), i32)
    pages = (cache, cache, table, starts, lens)
    split = (44, 42, 42)
    attn_of = B.dit_attn_paged_forward
    for call in (
            lambda: B.dit_qk_rope_forward(q, k, t((4, 3), f32), split), lambda: B.dit_qk_rope_forward(q, k, t((5, 3), i32), split),
            lambda: B.dit_qk_rope_forward(q, k, pos, (44, 42, 40)), lambda: B.dit_qk_rope_forward(q, k, pos, ((1 << 32) + 128, 0, 0)),
            lambda: B.dit_qk_rope_forward(q, t((4, 1, 128), f32), pos, split),
            lambda: B.dit_qk_rope_forward(q, k, pos, split, q_out=t((4, 3, 128)), k_out=k),
            lambda: B.dit_qk_rope_forward(q, None, pos, split, q_out=q, k_out=k),
            lambda: B.dit_qk_rope_forward(q, k, pos, split, q_out=q, k_out=t((4, 1, 128), f32)),
            lambda: B.dit_qk_rope_forward(q, k, pos, split, q_out=t((4, 2, 128), torch.float64), k_out=k),
            lambda: B.dit_qk_rope_forward(q, k, t((4, 3), i32, 1), split, q_out=q, k_out=k),
            lambda: B.dit_qk_rope_forward(q, k, pos, split, q_out=q, k_out=k, norm=("rows", 1e-6, None, None)),
            lambda: B.dit_qk_rope_forward(q, k, pos, split, q_out=q, k_out=k, norm=("head", 1e-6, t((128,), f32), None)),
            lambda: B.dit_qk_rope_forward(q, k, pos, split, q_out=q, k_out=k, norm=("head", 1e-6, None, t((128,), f32, 1))),
            lambda: B.dit_qk_rope_forward(t((4, 128, 2)).transpose(1, 2), None, pos, split, q_out=q),
            lambda: B.dit_kv_append_forward(k, k, cache, t((3, 16, 1, 128), torch.float16), table, starts, lens),
            lambda: B.dit_kv_append_forward(k, k, cache, t((3, 1, 16, 128)).transpose(1, 2)[:, :, :, :], t((2, 3), f32), starts, lens),
            lambda: B.dit_kv_append_forward(k, k, cache, cache, table, t((2,), i32), lens),
            lambda: B.dit_kv_append_forward(k, k, cache, cache, table, starts, t((3,), i32)),
            lambda: B.dit_kv_append_forward(k, k, t((3, 16, 1, 128), f32), t((3, 16, 1, 128), f32), table, starts, lens),
            lambda: B.dit_kv_append_forward(k, t((4, 1, 128), f32), *pages), lambda: B.dit_kv_append_forward(t((4, 2, 128)), q, *pages),
            lambda: B.dit_kv_append_forward(k, k, *pages, q_out=q), lambda: B.dit_kv_append_forward(k, k, *pages, q=q, q_out=t((4, 1, 128))),
            lambda: B.dit_kv_append_forward(k, k, *pages, pos=t((4, 2), i32), split=split),
            lambda: B.dit_kv_append_forward(k, k, t((3, 16, 1, 128), bf, 1), cache, table, starts, lens),
            lambda: attn_of(q, t((3, 16, 1, 64)), t((3, 16, 1, 64)), table, starts, lens),
            lambda: attn_of(t((4, 3, 128)), t((3, 16, 2, 128)), t((3, 16, 2, 128)), table, starts, lens),
            lambda: attn_of(q, *pages, out=t((4, 2, 128), torch.float16)), lambda: attn_of(q, *pages, out=t((3, 2, 128))),
            lambda: attn_of(q, *pages, out=q, lse=t((4, 2), f32)), lambda: attn_of(q, *pages, out=q, lse=t((2, 4))),
            lambda: attn_of(q, *pages, out=q, lse=t((2, 4), f32, 1)), lambda: attn_of(t((4, 2, 128), bf, 1), *pages)):
        with pytest.raises((ValueError, TypeError)):
            call()


def test_packed_parameters_are_the_structs():
    """The wrappers pack the parameters as bytes: every field where the struct has it."""
    ints = list(range(1, 100))
    take = iter(ints)

    def fields(c):
        out = []
        for name, kind in c._fields_:
            out += fields(kind) if hasattr(kind, "_fields_") else [float(next(take)) if kind is ctypes.c_float else next(take)]
        return out

    for c, pack in ((B.dit_qk_rope_params, B._ROPE_PACK), (B.dit_kv_append_params, B._APPEND_PACK),
                    (B.dit_paged_attn_params, B._PAGED_PACK)):
        take = iter(ints)
        values = fields(c)
        packed = pack(*values)
        got = c.from_buffer_copy(packed.ljust(ctypes.sizeof(c), b"\0"))
        assert len(packed) == ctypes.sizeof(c)
        flat = []

        def walk(x):
            for name, kind in x._fields_:
                v = getattr(x, name)
                walk(v) if hasattr(kind, "_fields_") else flat.append(v)

        walk(got)
        assert flat == values


def test_current_device_has_to_be_the_tensors(monkeypatch):
    import torch

    monkeypatch.setattr(B, "_stream_ptr", lambda stream: 7)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    assert B._stream_on("x", None, 1) == 7
    with pytest.raises(ValueError, match="device 0"):
        B._stream_on("x", None, 0)
    assert B._stream_on("x", SimpleNamespace(device_index=1), 1) == 7
    with pytest.raises(ValueError, match="stream"):
        B._stream_on("x", SimpleNamespace(device_index=0), 1)


def test_struct_layout(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not found")
    structs = ("dit_qk_rope_params", "dit_kv_cache", "dit_kv_append_params", "dit_paged_attn_params")
    src = tmp_path / "t.c"
    src.write_text('#include "dit_attn.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) {\n' + "".join(
        '  printf("%%zu", sizeof(%s));\n' % s + "".join(
            '  printf(" %%zu", offsetof(%s, %s));\n' % (s, f[0]) for f in getattr(B, s)._fields_) + '  printf("\\n");\n'
        for s in structs) + "  return 0;\n}\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o",
                           str(tmp_path / "t")])
    lines = subprocess.check_output([str(tmp_path / "t")], text=True).splitlines()
    for s, line in zip(structs, lines):
        c = getattr(B, s)
        assert [int(x) for x in line.split()] == [ctypes.sizeof(c)] + [getattr(c, f[0]).offset for f in c._fields_], s


@pytest.mark.parametrize("d", [1, 2, 3, 5, 7, 48, 64, 100, 1560, 2 ** 31 - 1, 2 ** 30 + 1, 2 ** 30, 641, 65537])
def test_division_by_a_product(d):
    """The multiplier and shift that the kernels divide by page sizes, frames and groups with: n / d for every n below 2^31 at
    which the quotient changes, and the ends."""
    import numpy as np

    l = 0
    while (1 << l) < d:
        l += 1
    mul = ((1 << (31 + l)) + d - 1) // d
    assert mul < 1 << 32
    rng = np.random.default_rng(d)
    n = [0, 1, 2 ** 31 - 1, 2 ** 31 - 2] + [int(x) for x in rng.integers(0, 2 ** 31, size=2000)]
    n += [x for q in rng.integers(0, max(1, (2 ** 31 - 1) // d), size=2000) for x in (int(q) * d - 1, int(q) * d) if x >= 0]
    for x in n:
        assert (((2 * x) & 0xffffffff) * mul >> 32) >> l == x // d
