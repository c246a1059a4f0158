"""Refusals and workspace sizes of the scored attention, the drafted-token attention and
the cache's keep, without a GPU: every call fails host-side validation (or has nothing
to do), so nothing is launched."""

import ctypes
import types

import pytest
import torch

from paper_2606_21848_amd import binding as kb
from tests.test_abi import FAKE, cache, expect, lib  # noqa: F401

ODD = ctypes.c_void_p(0x100008)


def desc(cap=0.0, slopes=None, first=None, last=None, causal=1):
    return kb.KLScoring(cap, slopes, first, last, causal)


def fwd(lib, sc=None, q=FAKE, v=FAKE, B=1, N=16, H=4, G=2, d=64, scale=0.0, dt=kb.KL_BF16, out=FAKE, lse=None,
        o32=None, null=False):
    sc = desc() if sc is None else sc
    return lib.keyless_scored_forward(q, v, None if null else ctypes.byref(sc), B, N, H, G, d, scale, dt, out,
                                      lse, o32, None)


def bwd(lib, sc=None, q=FAKE, v=FAKE, out=FAKE, o32=None, dout=FAKE, lse=FAKE, B=1, N=16, H=4, G=2, d=64,
        scale=0.0, dt=kb.KL_BF16, dq=FAKE, dv=FAKE, ws=FAKE, ws_bytes=1 << 40):
    sc = desc() if sc is None else sc
    return lib.keyless_scored_backward(q, v, out, o32, dout, lse, ctypes.byref(sc), B, N, H, G, d, scale, dt, dq,
                                       dv, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_scored_rejects_bad_arguments(lib, call):  # noqa: F811
    for kw in ("q", "v", "out"):
        expect(lib, call(lib, **{kw: None}), kb.KL_ERR_INVALID_ARG, "non-NULL")
        expect(lib, call(lib, **{kw: ODD}), kb.KL_ERR_INVALID_ARG, "aligned")
    expect(lib, call(lib, o32=ODD), kb.KL_ERR_INVALID_ARG, "aligned")
    expect(lib, call(lib, G=3), kb.KL_ERR_INVALID_ARG, "multiple")
    expect(lib, call(lib, d=96), kb.KL_ERR_UNSUPPORTED, "d_head 96")
    expect(lib, call(lib, dt=7), kb.KL_ERR_UNSUPPORTED, "dtype")
    expect(lib, call(lib, N=-1), kb.KL_ERR_INVALID_ARG, "bad sizes")
    expect(lib, call(lib, B=-1), kb.KL_ERR_INVALID_ARG, "bad sizes")
    expect(lib, call(lib, B=1 << 16, N=1 << 15), kb.KL_ERR_UNSUPPORTED, "too large")
    expect(lib, call(lib, N=1 << 28, H=256), kb.KL_ERR_UNSUPPORTED, "too large")
    expect(lib, call(lib, H=1 << 18, G=1), kb.KL_ERR_UNSUPPORTED, "2^24")
    for x in (-1.0, float("nan"), float("inf")):
        expect(lib, call(lib, scale=x), kb.KL_ERR_INVALID_ARG, "scale")
        expect(lib, call(lib, sc=desc(cap=x)), kb.KL_ERR_INVALID_ARG, "cap")
    assert call(lib, B=0) == kb.KL_OK and call(lib, N=0) == kb.KL_OK


def test_scored_rejects_the_rest(lib):  # noqa: F811
    expect(lib, fwd(lib, null=True), kb.KL_ERR_INVALID_ARG, "scoring")
    for kw in ("dout", "lse", "dq", "dv"):
        expect(lib, bwd(lib, **{kw: None}), kb.KL_ERR_INVALID_ARG, "non-NULL")
    for kw in ("dout", "dq", "dv", "ws"):
        expect(lib, bwd(lib, **{kw: ODD}), kb.KL_ERR_INVALID_ARG, "aligned")
    for dt in (kb.KL_BF16, kb.KL_F32):
        need = lib.keyless_scored_backward_workspace_size(2, 100, 4, 2, 64, dt)
        assert need >= 2 * 4 * 100 * 4
        expect(lib, bwd(lib, B=2, N=100, dt=dt, ws_bytes=need - 1), kb.KL_ERR_WORKSPACE, "workspace")
        expect(lib, bwd(lib, B=2, N=100, dt=dt, ws=None), kb.KL_ERR_WORKSPACE, "workspace")
    size = lib.keyless_scored_backward_workspace_size
    assert size(0, 9, 4, 2, 64, 0) == size(1, 9, 4, 3, 64, 0) == size(-1, 9, 4, 2, 64, 0) == 0


def tree(lib, c=None, q=FAKE, n=FAKE, words=FAKE, B=2, T=4, H=8, cap=0.0, scale=0.0, out=FAKE, ws=FAKE,
         ws_bytes=1 << 40):
    c = cache() if c is None else c
    return lib.keyless_tree_decode(q, ctypes.byref(c), n, words, B, T, H, cap, None, scale, out, ws, ws_bytes, None)


def test_tree_rejects_bad_arguments(lib):  # noqa: F811
    for kw in ("q", "n", "out"):
        expect(lib, tree(lib, **{kw: None}), kb.KL_ERR_INVALID_ARG, "non-NULL")
    for kw in ("q", "out"):
        expect(lib, tree(lib, **{kw: ODD}), kb.KL_ERR_INVALID_ARG, "aligned")
    expect(lib, tree(lib, words=ctypes.c_void_p(0x100004)), kb.KL_ERR_INVALID_ARG, "aligned")
    for T in (0, -1, 65):
        expect(lib, tree(lib, T=T), kb.KL_ERR_UNSUPPORTED, "drafted tokens")
    expect(lib, tree(lib, H=12), kb.KL_ERR_INVALID_ARG, "multiple")
    expect(lib, tree(lib, H=0), kb.KL_ERR_INVALID_ARG, "H=0")
    expect(lib, tree(lib, B=-1), kb.KL_ERR_INVALID_ARG, "B=-1")
    expect(lib, tree(lib, c=cache(d=96)), kb.KL_ERR_UNSUPPORTED, "d_head 96")
    expect(lib, tree(lib, c=cache(L_max=2 ** 31 - 1)), kb.KL_ERR_UNSUPPORTED, "capacity")
    expect(lib, tree(lib, B=1 << 24, T=64), kb.KL_ERR_UNSUPPORTED, "too large")
    expect(lib, tree(lib, B=1 << 16, T=4, H=8), kb.KL_ERR_UNSUPPORTED, "too large")
    expect(lib, tree(lib, c=cache(L_max=1 << 30), B=32, T=1), kb.KL_ERR_UNSUPPORTED, "too large")
    c = cache(L_max=5000)
    for B in (2, 9):
        need = lib.keyless_tree_decode_workspace_size(ctypes.byref(c), B, 4, 8)
        assert need > 0
        expect(lib, tree(lib, c=c, B=B, ws_bytes=need - 1), kb.KL_ERR_WORKSPACE, "workspace")
        expect(lib, tree(lib, c=c, B=B, ws=None), kb.KL_ERR_WORKSPACE, "workspace")
        expect(lib, tree(lib, c=c, B=B, ws=ODD), kb.KL_ERR_INVALID_ARG, "aligned")
    for x in (-1.0, float("nan"), float("inf")):
        expect(lib, tree(lib, cap=x), kb.KL_ERR_INVALID_ARG, "cap")
        expect(lib, tree(lib, scale=x), kb.KL_ERR_INVALID_ARG, "scale")
    assert lib.keyless_tree_decode(FAKE, None, FAKE, None, 1, 1, 1, 0.0, None, 0.0, FAKE, None, 0, None) == \
        kb.KL_ERR_INVALID_ARG
    assert tree(lib, B=0) == kb.KL_OK


def test_keep_rejects_bad_arguments(lib):  # noqa: F811
    c = cache()

    def keep(c=c, n=FAKE, path=FAKE, kept=FAKE, B=2, T=4):
        return lib.value_cache_keep(ctypes.byref(c), n, path, kept, B, T, None)
    for kw in ("n", "path", "kept"):
        expect(lib, keep(**{kw: None}), kb.KL_ERR_INVALID_ARG, "non-NULL")
    expect(lib, keep(T=65), kb.KL_ERR_UNSUPPORTED, "drafted tokens")
    expect(lib, keep(T=-1), kb.KL_ERR_INVALID_ARG, "T=-1")
    expect(lib, keep(B=-1), kb.KL_ERR_INVALID_ARG, "B=-1")
    expect(lib, keep(c=cache(layout=kb.KL_PAGED, bs=8)), kb.KL_ERR_UNSUPPORTED, "block_size")
    assert keep(B=0) == keep(T=0) == kb.KL_OK


def test_binding_checks_shapes_and_types(lib):  # noqa: F811
    """Tensors off the GPU, and descriptors that do not fit, are refused by the binding."""
    x = torch.zeros((1, 4, 2, 64))
    with pytest.raises(ValueError):
        kb.keyless_scored_forward(x, x, kb.Scoring())
    with pytest.raises(ValueError):
        kb.Scoring(slopes=torch.zeros(2))
    for shape, dtype, err in (((3,), torch.int32, ValueError), ((2, 2), torch.int64, TypeError)):
        with pytest.raises(err):
            kb._like(torch.zeros(shape, dtype=dtype), (2, 2), torch.int32, -1, "first")
    with pytest.raises(ValueError):
        kb._like(torch.zeros((2, 2), dtype=torch.int32), (2, 2), torch.int32, 0, "first")


def test_caps_that_fp32_or_bf16_cannot_hold(lib):  # noqa: F811
    """A cap that overflows scale / cap, and in bf16 one whose rounding would show."""
    for call in (lambda cap, dt: fwd(lib, sc=desc(cap=cap), dt=dt, N=0),
                 lambda cap, dt: bwd(lib, sc=desc(cap=cap), dt=dt, N=0),
                 lambda cap, dt: tree(lib, c=cache(dtype=dt), cap=cap, B=0)):
        for dt in (kb.KL_BF16, kb.KL_F32):
            expect(lib, call(1e-39, dt), kb.KL_ERR_UNSUPPORTED, "too small")
            assert call(1e-30, dt) == call(1024.0, dt) == kb.KL_OK
        expect(lib, call(1025.0, kb.KL_BF16), kb.KL_ERR_UNSUPPORTED, "at most 1024")
        assert call(3e38, kb.KL_F32) == kb.KL_OK


def test_binding_refuses_another_device():
    """A cache or a workspace that is not where the first argument is."""
    here = types.SimpleNamespace(data=torch.zeros((2, 1, 8, 64)), block_table=None, dev=-1)
    n = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="another device"):
        kb._per_sequence(here, n, 2, 0, "lengths_before")
    with pytest.raises(ValueError, match="2 sequences"):
        kb._per_sequence(here, n, 3, -1, "lengths_before")
    with pytest.raises(ValueError, match="another device"):
        kb._workspace(torch.zeros(256, dtype=torch.uint8), 0)
