"""Refusals of the dense sublayer's entry points, on the host before any HIP
call (no GPU needed; addresses are never dereferenced)."""

import ctypes

import pytest
import torch

import paper_2511_11505_amd as fs
from paper_2511_11505_amd import _lib as L

A, B, C, D, E = ((1 << 30) * (i + 1) for i in range(5))   # far apart, aligned, not memory
BIG = (1 << 29, 1 << 60)                                   # a workspace address and size


def refuse(status, text, fn, *args, **kw):
    if "workspace" not in fn.__name__:
        kw["stream"] = 0
    with pytest.raises(L.FsError) as e:
        fn(*args, **kw)
    assert e.value.status == status, str(e.value)
    assert text in str(e.value), str(e.value)


def lin(m=8, n=16, k=24, act="none", **kw):
    d = fs.linear_desc(m, n, k, "bf16", act if isinstance(act, str) else "none")
    d.act = d.act if isinstance(act, str) else act
    for f, v in kw.items():
        setattr(d, f, v)
    return d


@pytest.mark.parametrize("kw,status", [
    (dict(abi_version=1), L.FS_ERR_INVALID), (dict(dtype=2), L.FS_ERR_INVALID),
    (dict(act=4), L.FS_ERR_INVALID), (dict(act=-1), L.FS_ERR_INVALID), (dict(m=-1), L.FS_ERR_INVALID),
    (dict(n=0), L.FS_ERR_INVALID), (dict(k=0), L.FS_ERR_INVALID),
    (dict(m=2 ** 24 + 1), L.FS_ERR_UNSUPPORTED), (dict(n=2 ** 31 - 1), L.FS_ERR_UNSUPPORTED),
    (dict(m=2 ** 20, n=2 ** 20), L.FS_ERR_UNSUPPORTED)])
def test_linear_descriptor(kw, status):
    d = lin(**kw)
    refuse(status, "", fs.fs_linear, d, A, B, None, None, C, BIG)
    refuse(status, "", fs.fs_linear_workspace, d, L.FS_OP_LINEAR)
    refuse(status, "", fs.fs_linear_backward, d, A, B, C, None, D, E, None, BIG)


def test_linear_arguments():
    d = lin()
    refuse(L.FS_ERR_INVALID, "a must not be NULL", fs.fs_linear, d, None, B, None, None, C, BIG)
    refuse(L.FS_ERR_INVALID, "w must not be NULL", fs.fs_linear, d, A, None, None, None, C, BIG)
    refuse(L.FS_ERR_INVALID, "out must not be NULL", fs.fs_linear, d, A, B, None, None, None, BIG)
    refuse(L.FS_ERR_INVALID, "aligned", fs.fs_linear, d, A + 1, B, None, None, C, BIG)
    refuse(L.FS_ERR_INVALID, "bias", fs.fs_linear, d, A, B, D + 2, None, C, BIG)
    refuse(L.FS_ERR_INVALID, "overlap", fs.fs_linear, d, A, B, None, None, A + 8 * 24 * 2 - 2, BIG)
    refuse(L.FS_ERR_INVALID, "overlap", fs.fs_linear, d, A, B, None, C + 2, C, BIG)
    refuse(L.FS_ERR_INVALID, "overlap", fs.fs_linear, d, A, B, None, None, C, BIG, save_z=C)
    refuse(L.FS_ERR_INVALID, "neither", fs.fs_linear, d, A, B, None, None, C, BIG, save_z=L.fs_saved())
    refuse(L.FS_ERR_INVALID, "codes only", fs.fs_linear, d, A, B, None, None, C, BIG, save_out=D)
    refuse(L.FS_ERR_INVALID, "without scales", fs.fs_linear, d, A, B, None, None, C, BIG, save_z=(D, None))
    big = lin(1, 16, 4096)
    assert fs.fs_linear_workspace(big, L.FS_OP_LINEAR) > 0      # split over K
    refuse(L.FS_ERR_WORKSPACE, "fs_linear_workspace", fs.fs_linear, big, A, B, None, None, C, (D, 16))
    refuse(L.FS_ERR_INVALID, "ws must", fs.fs_linear, big, A, B, None, None, C, (D + 8, 1 << 60))
    refuse(L.FS_ERR_INVALID, "op must", fs.fs_linear_workspace, d, L.FS_OP_BLOCK)


def test_linear_row_strides():
    """A stride below the columns, as an expanded row has, is refused."""
    d, lib, ok = lin(), L.load(), (None, None)
    for i, (lda, ldw, ldr, ldo) in enumerate([(23, 24, 16, 16), (24, 0, 16, 16), (24, 24, 15, 16), (24, 24, 16, 1)]):
        st = lib.fs_linear(ctypes.byref(d), A, lda, B, ldw, None, D, ldr, C, ldo, *ok, None, 0, None)
        assert st == L.FS_ERR_INVALID, i
        assert b"row stride" in lib.fs_last_error_message()


def test_in_place_needs_the_same_stride():
    """An output on an input's base with another stride is refused."""
    lib, d, n = L.load(), lin(), norm()
    st = lib.fs_linear(ctypes.byref(d), A, 24, B, 24, None, C, 20, C, 16, None, None, None, 0, None)
    assert st == L.FS_ERR_INVALID and b"overlap" in lib.fs_last_error_message()
    st = lib.fs_layer_norm(ctypes.byref(n), A, 48, None, 0, None, None, None, 0, A, 40, None, None, None, None, None)
    assert st == L.FS_ERR_INVALID and b"overlap" in lib.fs_last_error_message()
    refuse(L.FS_ERR_INVALID, "overlap", fs.fs_linear, d, A, B, None, None, C, BIG, save_z=(C, D))
    refuse(L.FS_ERR_INVALID, "overlap", fs.fs_layer_norm, n, A, None, None, None, None, B, None, None,
           save_in=(A, C))


def test_linear_empty():
    for op in (L.FS_OP_LINEAR, L.FS_OP_LINEAR_BACKWARD):
        assert fs.fs_linear_workspace(lin(m=0, n=40, k=4096, act="gelu"), op) == 0
    fs.fs_linear(lin(m=0), None, None, None, None, None, None, stream=0)


def test_linear_backward_arguments():
    d, dz = lin(), lin(act="gelu")
    bwd = fs.fs_linear_backward
    refuse(L.FS_ERR_INVALID, "all NULL", bwd, d, A, B, C, None, None, None, None, BIG)
    refuse(L.FS_ERR_INVALID, "dout", bwd, d, None, B, C, None, D, E, None, BIG)
    refuse(L.FS_ERR_INVALID, "dw needs a", bwd, d, A, None, C, None, D, E, None, BIG)
    refuse(L.FS_ERR_INVALID, "w must not", bwd, d, A, B, None, None, D, E, None, BIG)
    refuse(L.FS_ERR_INVALID, "z must not", bwd, dz, A, B, C, None, D, E, None, BIG)
    refuse(L.FS_ERR_INVALID, "overlap", bwd, d, A, B, C, None, A + 2, E, None, BIG)
    refuse(L.FS_ERR_INVALID, "overlap", bwd, d, A, B, C, None, B, E, None, BIG)
    refuse(L.FS_ERR_INVALID, "overlap", bwd, d, A, B, C, None, D, D, None, BIG)
    refuse(L.FS_ERR_INVALID, "both rows and codes", bwd, d, A, L.fs_saved(B, 24, D, D), C, None, D, E, None, BIG)
    refuse(L.FS_ERR_WORKSPACE, "BACKWARD", bwd, dz, A, B, C, D, D + (1 << 20), E, None, (A, 16))


def norm(rows=4, cols=40, **kw):
    d = fs.norm_desc(rows, cols)
    for f, v in kw.items():
        setattr(d, f, v)
    return d


@pytest.mark.parametrize("kw,status", [
    (dict(abi_version=1), L.FS_ERR_INVALID), (dict(dtype=-1), L.FS_ERR_INVALID),
    (dict(rows=-1), L.FS_ERR_INVALID), (dict(cols=0), L.FS_ERR_INVALID),
    (dict(cols=32769), L.FS_ERR_UNSUPPORTED), (dict(rows=2 ** 21 + 1), L.FS_ERR_UNSUPPORTED),
    (dict(center=2), L.FS_ERR_INVALID), (dict(eps=0.0), L.FS_ERR_INVALID),
    (dict(eps=float("nan")), L.FS_ERR_INVALID), (dict(eps=float("inf")), L.FS_ERR_INVALID)])
def test_norm_descriptor(kw, status):
    d = norm(**kw)
    refuse(status, "", fs.fs_layer_norm, d, A, None, None, None, None, B, None, None)
    refuse(status, "", fs.fs_layer_norm_workspace, d)
    refuse(status, "", fs.fs_layer_norm_backward, d, A, B, C, D, None, None, E, None, None, None)


def test_norm_arguments():
    d, f, b = norm(), fs.fs_layer_norm, fs.fs_layer_norm_backward
    refuse(L.FS_ERR_INVALID, "x must not", f, d, None, None, None, None, None, B, None, None)
    refuse(L.FS_ERR_INVALID, "y must not", f, d, A, None, None, None, None, None, None, None)
    refuse(L.FS_ERR_INVALID, "overlap", f, d, A, None, None, None, None, A + 2, None, None)
    refuse(L.FS_ERR_INVALID, "overlap", f, d, A, None, None, None, B, B, None, None)
    refuse(L.FS_ERR_INVALID, "4-byte", f, d, A, None, C + 1, None, None, B, None, None)
    refuse(L.FS_ERR_INVALID, "codes only", f, d, A, None, None, None, None, B, None, None, save_y=C)
    refuse(L.FS_ERR_INVALID, "x must not", b, d, A, None, C, D, None, None, E, None, None, None)
    refuse(L.FS_ERR_INVALID, "rstd", b, d, A, B, C, None, None, None, E, None, None, None)
    refuse(L.FS_ERR_INVALID, "mean", b, d, A, B, None, D, None, None, E, None, None, None)
    refuse(L.FS_ERR_INVALID, "overlap", b, d, A, B, C, D, None, None, B, None, None, None)
    refuse(L.FS_ERR_WORKSPACE, "workspace", b, d, A, B, C, D, None, None, E, C, None, (A, 0))
    f(norm(rows=0), None, None, None, None, None, None, None, None, stream=0)


def test_checkpoint_arguments():
    enc, dec = fs.fs_checkpoint_fp8, fs.fs_checkpoint_restore
    refuse(L.FS_ERR_INVALID, "dtype", enc, 3, 4, 40, A, B, C)
    refuse(L.FS_ERR_INVALID, "cols", enc, L.FS_F32, 4, 0, A, B, C)
    refuse(L.FS_ERR_INVALID, "rows", dec, L.FS_F32, -1, 4, B, C, A)
    refuse(L.FS_ERR_INVALID, "codes and scales", enc, L.FS_F32, 4, 40, A, None, C)
    refuse(L.FS_ERR_INVALID, "src must not", enc, L.FS_F32, 4, 40, None, B, C)
    refuse(L.FS_ERR_INVALID, "aligned", enc, L.FS_F32, 4, 40, A + 2, B, C)
    refuse(L.FS_ERR_INVALID, "overlap", enc, L.FS_F32, 4, 40, A, A + 8, C)
    refuse(L.FS_ERR_INVALID, "overlap", dec, L.FS_BF16, 4, 40, B, C, C)
    enc(L.FS_F32, 0, 40, None, None, None, stream=0)


def test_binding_refuses_what_the_library_cannot_see():
    """Type, shape, layout and device of tensors."""
    d = lin()
    x = torch.zeros((8, 24), dtype=torch.bfloat16)
    refuse(L.FS_ERR_INVALID, "a must be [8, 24]", fs.fs_linear, d, x.float(), B, None, None, C, BIG)
    refuse(L.FS_ERR_INVALID, "a must be [8, 24]", fs.fs_linear, d, x[:7], B, None, None, C, BIG)
    refuse(L.FS_ERR_INVALID, "column stride", fs.fs_linear, d, x.t().contiguous().t(), B, None, None, C, BIG)
    refuse(L.FS_ERR_INVALID, "GPU", fs.fs_linear, d, x, B, None, None, C, BIG)
    refuse(L.FS_ERR_INVALID, "bias", fs.fs_linear, d, A, B, torch.zeros(8), None, C, BIG)
    refuse(L.FS_ERR_INVALID, "codes", fs.fs_linear, d, A, B, None, None, C, BIG,
           save_z=fs.checkpoint_buffers(8, 17, "cpu"))
    with pytest.raises(ValueError):
        fs.DenseSublayer(4, None, None, torch.zeros(6, 4), None, torch.zeros(6, 4), None)
    with pytest.raises(ValueError):
        fs.DenseSublayer(4, None, None, torch.zeros(6, 4), None, torch.zeros(4, 6), None, save="fp8")


def test_outputs_lie_apart():
    """Vectors, scale bytes, checkpoints and the workspace, too, lie apart from
    every input and from each other."""
    lib, d, big, n = L.load(), lin(), lin(1, 16, 4096), norm()
    fwd, bwd, ln, lnb = fs.fs_linear, fs.fs_linear_backward, fs.fs_layer_norm, fs.fs_layer_norm_backward
    INV, text = L.FS_ERR_INVALID, "overlap"
    refuse(INV, text, fwd, d, A, B, C, None, C, BIG)                                  # out, bias
    refuse(INV, text, fwd, d, A, B, None, None, C, BIG, save_z=(D, C))                # out, scales
    refuse(INV, text, fwd, d, A, B, None, None, C, BIG, save_z=(D, E), save_out=(D, E + 64))
    refuse(INV, text, fwd, d, A, B, None, None, C, BIG, save_z=(D, E), save_out=(D + 4096, E))
    refuse(INV, text, fwd, d, A, B, None, D, C, BIG, save_z=(D + 16, E))              # residual, codes
    refuse(INV, text, fwd, big, A, B, None, None, C, (B + 64, 1 << 60))               # w, ws
    refuse(INV, text, bwd, d, A, B, C, None, D, E, E + 4, BIG)                        # dw, dbias
    refuse(INV, text, bwd, d, A, (B, E), C, None, D, E, None, BIG)                    # dw, a's scales
    refuse(INV, text, bwd, lin(act="gelu"), A, B, C, D, E, None, None, (D, 1 << 60))  # z, ws
    refuse(INV, text, ln, n, A, None, None, None, None, B, C, C + 4)                  # mean, rstd
    refuse(INV, text, ln, n, A, None, B + 8, None, None, B, None, None)               # y, gamma
    refuse(INV, text, ln, n, A, None, None, None, None, A, None, None, save_y=(A, B))
    refuse(INV, text, lnb, n, A, B, C, D, None, None, E, E + 4, None, BIG)            # dx, dgamma
    refuse(INV, text, lnb, n, A, B, C, D, None, None, C, None, None, BIG)             # dx, mean
    refuse(INV, text, lnb, n, A, B, C, D, None, None, E, D, None, BIG)                # dgamma, rstd
    refuse(INV, text, lnb, n, A, B, C, D, None, None, E, E + 4096, None, (A, 1 << 60))
    # one row's stride says nothing about gaps
    one = lin(1)
    st = lib.fs_linear(ctypes.byref(one), A, 100, B, 24, None, None, 0, A + 40, 50, None, None, None, 0, None)
    assert st == INV and b"overlap" in lib.fs_last_error_message()


def test_binding_refuses_a_workspace_elsewhere():
    """A workspace on the host, or one whose bytes do not lie together."""
    d, n = lin(1, 16, 4096), norm()
    host, gaps = torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(1 << 20, dtype=torch.uint8)[::2]
    for ws, text in ((host, "ws must be on the current GPU"), (gaps, "ws must be contiguous")):
        refuse(L.FS_ERR_INVALID, text, fs.fs_linear, d, A, B, None, None, C, ws)
        refuse(L.FS_ERR_INVALID, text, fs.fs_linear_backward, d, A, B, C, None, D, E, None, ws)
        refuse(L.FS_ERR_INVALID, text, fs.fs_layer_norm_backward, n, A, B, C, D, None, None, E, E + 4096, None, ws)


@pytest.mark.parametrize("save", ["rows", "codes"])
def test_sublayer_backward_before_forward(save):
    """Nothing is saved yet, nor after a forward pass that was refused."""
    layer = sublayer(save)
    x = torch.zeros((3, 4), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="before forward"):
        layer.backward(x, {})
    with pytest.raises(L.FsError):
        layer.forward(x, torch.zeros((3, 5), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="before forward"):
        layer.backward(x, {})


def sublayer(save, tokens=3, d=4, f=6):
    w1, w2 = torch.zeros((f, d), dtype=torch.bfloat16), torch.zeros((d, f), dtype=torch.bfloat16)
    return fs.DenseSublayer(tokens, None, None, w1, None, w2, None, save=save)


def test_sublayer_in_place_would_lose_the_saved_rows():
    x = torch.zeros((3, 4), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="may not be x"):
        sublayer("rows").forward(x, x)


def held_bytes(layer):
    """Bytes of the distinct tensors that a sublayer keeps beside its
    parameters."""
    held = {}
    for v in vars(layer).values():
        for t in v if isinstance(v, tuple) else (v,):
            if isinstance(t, torch.Tensor) and not any(t is q for q in layer.params):
                held[t.untyped_storage().data_ptr()] = t.untyped_storage().nbytes()
    return sum(held.values())


@pytest.mark.parametrize("d,f", [(64, 64), (256, 256), (256, 1024), (512, 128)])
def test_sublayer_codes_hold_less_than_rows(d, f):
    """A token's bytes beyond the workspace, as documented."""
    n = 96
    rows, codes = sublayer("rows", n, d, f), sublayer("codes", n, d, f)
    stats = 2 * 4 * n   # mean, rstd
    assert held_bytes(rows) - rows.ws.numel() - stats == n * (4 * d + 6 * f)
    kept = n * (2 * (d + f) + 2 * (d + f) * 33 // 32)
    assert held_bytes(codes) - codes.ws.numel() - stats == kept
    # (rows mode reads the caller's x as well)
    assert kept < n * (4 * d + 6 * f + 2 * d)
