"""C-ABI checks of libspardl_train.so that need no GPU: every entry point of
include/spardl_train.h is exported, bound and refuses bad arguments before
anything is enqueued; no instruction pattern that took wrong values is in its
kernels."""

import ctypes
import os
import re
import subprocess

import pytest

from tests.test_codegen import CSRC, HIPCC, suspicious_selects
from tests.train_calls import calls

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2304_00737_amd", "libspardl_train.so")
HEADER = os.path.join(ROOT, "include", "spardl_train.h")
EINVAL, ECAP, OK = -1, -2, 0

needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libspardl_train.so not built")
P = 0x1000                      # never dereferenced: validation fails first, or there are no rows
BIG = 1 << 40
OPTIONAL = {"res", "sum", "dsum", "dx", "gate", "up"}      # None by themselves, in some of the calls


def _binding():
    from paper_2304_00737_amd import train
    return train, train._lib


def declared():
    return sorted(set(re.findall(r"^\s*(?:int|size_t)\s+(spardl_\w+)\s*\(", open(HEADER).read(), re.M)))


@needs_lib
def test_every_entry_point_is_exported_and_bound():
    names = declared()
    assert len(names) == 10
    train, lib = _binding()
    for n in names:
        assert getattr(lib, n).argtypes, n
        if not n.endswith("workspace_bytes"):
            assert callable(getattr(train, n[len("spardl_"):])), n


@needs_lib
def test_norm_refusals():
    _, lib = _binding()

    def fwd(x=P, ldx=8, res=P, ldr=8, w=P, s=P, lds=8, y=P, ldy=8, rstd=P, rows=4, dim=8, eps=1e-6, dt=0):
        return lib.spardl_rms_norm(x, ldx, res, ldr, w, s, lds, y, ldy, rstd, rows, dim, eps, dt, None)

    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(ldx=7), dict(ldr=7), dict(lds=7), dict(ldy=7),
                dict(rows=-1), dict(dim=0), dict(dim=16385, ldx=BIG, ldr=BIG, lds=BIG, ldy=BIG), dict(eps=-1e-6),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(dt=3), dict(dt=-1), dict(x=P + 1), dict(rstd=P + 2),
                dict(x=P + 2, dt=2)):
        assert fwd(**bad) == EINVAL, bad
    assert fwd(rows=1 << 30, ldx=1 << 31) == EINVAL       # a matrix past 2^60 elements
    assert fwd(rows=0) == OK and fwd(rows=0, x=None, y=None, res=None, s=None, rstd=None) == OK

    def bwd(dy=P, ld=8, s=P, w=P, rstd=P, ds=P, dx=P, dw=P, rows=4, dim=8, dt=0, ws=P, n=1 << 20):
        return lib.spardl_rms_norm_backward(dy, ld, s, ld, w, rstd, ds, ld, dx, ld, dw, rows, dim, dt, ws, n, None)

    for bad in (dict(dy=None), dict(s=None), dict(w=None), dict(rstd=None), dict(dx=None), dict(dw=None), dict(ws=None),
                dict(ws=P + 16), dict(ld=7), dict(rows=-1), dict(dim=0), dict(dt=3), dict(dw=P + 1)):
        assert bwd(**bad) == EINVAL, bad
    assert bwd(n=8) == ECAP
    assert lib.spardl_rms_norm_workspace_bytes(-1, 8) == 0 and lib.spardl_rms_norm_workspace_bytes(5, 16385) == 0
    assert lib.spardl_rms_norm_workspace_bytes(5, 8) >= 5 * 8 * 4


@needs_lib
def test_distill_refusals():
    _, lib = _binding()

    def call(which, z=P, ld=100, i=P, v=P, ldt=4, rows=3, vocab=100, top=4, t=1.0, loss=P, stats=P, dl=P, d=P, ldd=100,
             dt=0, ws=P, n=1 << 20):
        if which == "loss":
            return lib.spardl_distill_loss(z, ld, i, v, ldt, rows, vocab, top, t, loss, stats, dt, ws, n, None)
        if which == "backward":
            return lib.spardl_distill_backward(z, ld, i, v, ldt, stats, dl, rows, vocab, top, t, d, ldd, dt, None)
        return lib.spardl_distill_loss_backward(z, ld, i, v, ldt, dl, rows, vocab, top, t, loss, stats, d, ldd, dt, ws,
                                                n, None)

    common = [dict(z=None), dict(i=None), dict(v=None), dict(stats=None), dict(ld=99), dict(ldt=3), dict(rows=-1),
              dict(vocab=0), dict(top=0), dict(top=1025, ldt=2000), dict(t=0.0), dict(t=-1.0), dict(t=float("nan")),
              dict(t=float("inf")), dict(dt=3), dict(z=P + 1), dict(i=P + 2)]
    ws = [dict(ws=None), dict(ws=P + 64), dict(loss=None)]
    grad = [dict(dl=None), dict(d=None), dict(ldd=99), dict(d=P + 1)]
    for which, more in (("loss", ws), ("backward", grad), ("both", ws + grad)):
        for bad in common + more:
            assert call(which, **bad) == EINVAL, (which, bad)
        assert call(which, rows=0) == OK
    assert call("loss", n=4) == ECAP and call("both", n=4) == ECAP
    assert lib.spardl_distill_workspace_bytes(-1, 8) == 0 and lib.spardl_distill_workspace_bytes(1, 0) == 0


@needs_lib
@pytest.mark.parametrize("t", [2.0 ** -127, 2.0 ** -149, -2.0 ** -127, -0.0, float("-inf")])
def test_distill_refuses_a_temperature_without_a_finite_reciprocal(t):
    _, lib = _binding()
    assert lib.spardl_distill_loss(P, 100, P, P, 4, 3, 100, 4, t, P, P, 0, P, 1 << 20, None) == EINVAL
    assert lib.spardl_distill_backward(P, 100, P, P, 4, P, P, 3, 100, 4, t, P, 100, 0, None) == EINVAL
    assert lib.spardl_distill_loss_backward(P, 100, P, P, 4, P, 3, 100, 4, t, P, P, P, 100, 0, P, 1 << 20, None) == EINVAL
    assert lib.spardl_distill_loss(P, 100, P, P, 4, 0, 100, 4, 2.0 ** -126, P, P, 0, P, 1 << 20, None) == OK


@needs_lib
def test_ffn_refusals():
    _, lib = _binding()

    def fwd(x=P, ldx=64, g=P, u=P, ldw=64, d=P, ldd=128, y=P, ldy=64, gate=P, up=P, ldh=128, T=3, D=64, F=128, act=0,
            dt=0, ws=P, n=1 << 30):
        return lib.spardl_gated_ffn(x, ldx, g, ldw, u, ldw, d, ldd, y, ldy, gate, up, ldh, T, D, F, act, dt, ws, n, None)

    common = [dict(x=None), dict(g=None), dict(u=None), dict(d=None), dict(ldx=63), dict(ldw=63), dict(ldd=127),
              dict(ldh=127), dict(T=-1), dict(D=0), dict(F=0), dict(T=1 << 31), dict(D=(1 << 20) + 1), dict(act=2),
              dict(act=-1), dict(dt=2), dict(dt=7), dict(gate=None), dict(up=None), dict(ws=None), dict(ws=P + 128),
              dict(x=P + 1)]
    for bad in common + [dict(y=None), dict(ldy=63)]:
        assert fwd(**bad) == EINVAL, bad
    assert fwd(n=100) == ECAP
    big = dict(ldx=1 << 20, ldw=1 << 20, ldd=1 << 20, ldy=1 << 20, ldh=1 << 20, n=1 << 60)
    assert fwd(T=1 << 30, D=128, F=64, **big) == EINVAL and fwd(T=1, D=1 << 19, F=1 << 19, **big) == EINVAL
    small, large = (lib.spardl_gated_ffn_workspace_bytes(3, 64, 128, 0, a) for a in (0, 1))
    assert 0 < small < large
    assert fwd(x=P + 2, n=small) == ECAP and fwd(ldw=65, n=small) == ECAP       # no room for aligned copies
    assert fwd(T=0) == OK and fwd(T=0, x=None, y=None, gate=None, up=None) == OK

    def bwd(dy=P, x=P, gate=P, up=P, ldh=128, g=P, u=P, ldw=64, d=P, ldd=128, ldx=64, dx=P, dg=P, du=P, dd=P, lddw=64,
            dwt=0, T=3, D=64, F=128, act=0, dt=0, ws=P, n=1 << 30):
        return lib.spardl_gated_ffn_backward(dy, ldx, x, ldx, gate, up, ldh, g, ldw, u, ldw, d, ldd, dx, ldx, dg, lddw, du,
                                             lddw, dd, 128, dwt, 0, T, D, F, act, dt, ws, n, None)

    for bad in common + [dict(dy=None), dict(dg=None), dict(du=None), dict(dd=None), dict(lddw=63), dict(dwt=1),
                         dict(dwt=3), dict(gate=None, up=None), dict(dg=P + 2, dwt=2)]:
        assert bwd(**bad) == EINVAL, bad
    assert bwd(n=100) == ECAP
    assert lib.spardl_gated_ffn_workspace_bytes(3, 0, 8, 0, 0) == 0


@needs_lib
@pytest.mark.parametrize("dim,hidden", [(1600, 6400), (4096, 11008), (1001, 2731), (256, 704), (64, 64), (1, 1)])
def test_ffn_workspace_of_a_batch_serves_smaller_ones(dim, hidden):
    _, lib = _binding()
    for backward in (0, 1):
        for unaligned in (0, 1):
            last = 0
            for tokens in [*range(0, 2100), *range(2100, 20000, 7)]:
                now = lib.spardl_gated_ffn_workspace_bytes(tokens, dim, hidden, backward, unaligned)
                assert now >= last, (tokens, backward, unaligned, last, now)
                last = now


@needs_lib
def test_few_tokens_need_no_copies_of_odd_weights():
    _, lib = _binding()
    size = lib.spardl_gated_ffn_workspace_bytes
    for tokens in (0, 1, 2, 16):
        for dim, hidden in ((4097, 11009), (4096, 11009), (4097, 11008), (4096, 11008)):
            assert size(tokens, dim, hidden, 0, 0) <= 2 * tokens * 11016 + 512
    assert size(17, 4097, 11009, 0, 0) >= size(1, 4096, 11008, 0, 1) >= 6 * 4096 * 11008     # with copies


@needs_lib
def test_row_workspaces_of_a_batch_serve_smaller_ones():
    _, lib = _binding()
    rows = [*range(0, 3000), *range(3000, 70000, 61)]
    for vocab in (1, 2048, 2049, 8193, 50257, 131072, 1 << 30):
        sizes = [lib.spardl_distill_workspace_bytes(r, vocab) for r in rows]
        assert sizes == sorted(sizes) and sizes[0] > 0, vocab
    for dim in (1, 64, 1001, 4096, 16384):
        sizes = [lib.spardl_rms_norm_workspace_bytes(r, dim) for r in rows]
        assert sizes == sorted(sizes) and sizes[0] > 0, dim


@needs_lib
def test_python_refusals():
    import torch
    train, _ = _binding()
    e = torch.empty
    with pytest.raises(train.SpardlError, match="contiguous rows"):
        train.rms_norm(e(4, 8), e(4, 9), e(8), None, e(4, 8), stream=0)
    with pytest.raises(train.SpardlError, match="contiguous rows"):
        train.rms_norm(e(8, 4).t(), None, e(8), None, e(4, 8), stream=0)
    with pytest.raises(train.SpardlError, match="no kernel for"):
        train.rms_norm(e(4, 8).double(), None, e(8).double(), None, e(4, 8).double(), stream=0)
    with pytest.raises(train.SpardlError, match="contiguous rows"):
        train.distill_loss(e(2, 9), e(2, 3), e(2, 3), e(2), e(2, 2), None, stream=0)      # tokens in float
    with pytest.raises(train.SpardlError, match="act must be"):
        train.gated_ffn(e(2, 8).half(), e(4, 8).half(), e(4, 8).half(), e(8, 4).half(), e(2, 8).half(), None, act="relu",
                        stream=0)
    with pytest.raises(train.SpardlError) as err:
        train.gated_ffn(e(2, 8), e(4, 8), e(4, 8), e(8, 4), e(2, 8), e(256), stream=0)    # fp32
    assert err.value.status == EINVAL


@needs_lib
def test_workspaces_with_gaps_are_refused():
    """A view's elements times their size are not what lies behind its pointer."""
    train, _ = _binding()
    for name, tensors in calls("cpu"):
        if "ws" in tensors:
            for ws in (tensors["ws"][::2], tensors["ws"][:1].expand(1 << 20)):
                with pytest.raises(train.SpardlError, match="must be contiguous") as err:
                    getattr(train, name)(**{**tensors, "ws": ws}, stream=0)
                assert err.value.status == EINVAL


@needs_lib
def test_arguments_that_are_no_matrices_are_refused():
    """Missing, one-dimensional and three-dimensional arguments: an error of this library, whichever they are."""
    train, _ = _binding()
    for name, tensors in calls("cpu"):
        for arg, t in tensors.items():
            if t.ndim == 2:
                for other in (None, t[0], t[None]) if arg not in OPTIONAL else (t[0], t[None]):
                    with pytest.raises(train.SpardlError) as err:
                        getattr(train, name)(**{**tensors, arg: other}, stream=0)
                    assert err.value.status == EINVAL, (name, arg)


@needs_lib
def test_host_tensors_are_refused():
    """A host tensor's pointer never reaches a kernel; the shapes, types and sizes are all as they should be."""
    train, _ = _binding()
    for name, tensors in calls("cpu"):
        for stream in (None, 0):
            with pytest.raises(train.SpardlError, match="current GPU") as err:
                getattr(train, name)(**tensors, stream=stream)
            assert err.value.status == EINVAL


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
@pytest.mark.parametrize("src", ["train_norm.hip", "train_distill.hip", "train_ffn_bf16.hip", "train_ffn_fp16.hip"])
def test_no_select_reads_a_carry(tmp_path, src):
    from paper_2304_00737_amd import build
    assert src in build.TRAIN_SOURCES and len(build.TRAIN_SOURCES) == 5
    asm = tmp_path / (src + ".s")
    flags = [f for f in build.HIP_FLAGS if f not in ("-fPIC", "-shared", "-Wall")]
    subprocess.run([HIPCC, *flags, "--cuda-device-only", "-S", os.path.join(CSRC, src), "-o", str(asm)], check=True,
                   capture_output=True, timeout=600)
    text = asm.read_text()
    bad = suspicious_selects(text)
    assert not bad, "\n".join(bad[:10])
    assert not re.findall(r"v_pk_(?:add|mul|fma)_f32", text)
