"""The dense sublayer that runs in the far-skip window, and its gradient.

FarSkip runs the next layer's dense computation between the block's BEGIN and
FINISH phases, on an input that lacks the block's routed output (Section 3,
Eq. 8b).  ``DenseSublayer`` is that computation in full:

    h = norm(x);  u = act(h w1^T + b1);  out = x + u w2^T + b2

forward and backward, through fs_layer_norm, fs_linear and their backward
passes.  With ``save="codes"`` the activations that the backward pass reads (x,
h, the pre-activation and u) are kept as 8-bit checkpoints, written by the
passes that compute them, and the rows of h and u, read no more after the
forward pass, become those of their gradients: in bf16 4.1 (d + f) bytes a
token, against 4 d + 6 f and the caller's x with "rows", which keeps them as
they are; with None (serving) nothing is kept.  All arithmetic runs in the library's kernels; torch only allocates
memory.  A sublayer's passes share its buffers and its workspace, so they run
one after another, on one stream or ordered by events.
"""

import torch

from . import _lib as L

_TYPES = {"f32": (L.FS_F32, torch.float32), "bf16": (L.FS_BF16, torch.bfloat16)}
_ACTS = {"none": L.FS_ACT_NONE, "relu": L.FS_ACT_RELU, "gelu": L.FS_ACT_GELU, "silu": L.FS_ACT_SILU}


def linear_desc(m, n, k, dtype="bf16", act="none"):
    """fs_linear_desc of m tokens, n outputs, k inputs."""
    return L.fs_linear_desc(L.FS_ABI_VERSION, _TYPES[dtype][0], _ACTS[act], m, n, k)


def norm_desc(rows, cols, dtype="bf16", center=True, eps=1e-5):
    """fs_norm_desc of a layer norm (center) or root-mean-square norm."""
    return L.fs_norm_desc(L.FS_ABI_VERSION, _TYPES[dtype][0], rows, cols, int(center), eps)


def checkpoint_buffers(rows, cols, device="cuda"):
    """Codes and scales for an 8-bit checkpoint of [rows, cols]."""
    return (torch.empty((rows, cols), dtype=torch.uint8, device=device),
            torch.empty((rows, (cols + 31) // 32), dtype=torch.uint8, device=device))


class DenseSublayer:
    def __init__(self, tokens, gamma, beta, w1, b1, w2, b2, act="silu", center=True, eps=1e-5,
                 save=None):
        """gamma, beta [d] fp32 or None; w1 [f, d], w2 [d, f] bf16 or fp32;
        b1 [f], b2 [d] fp32 or None.  save: None, "rows" or "codes"."""
        if save not in (None, "rows", "codes"):
            raise ValueError(f"save must be None, 'rows' or 'codes', not {save!r}")
        f, d = w1.shape
        if tuple(w2.shape) != (d, f):
            raise ValueError(f"w2 must be [{d}, {f}], not {list(w2.shape)}")
        dtype = "f32" if w1.dtype == torch.float32 else "bf16"
        dt, dev = _TYPES[dtype][1], w1.device
        self.params = (gamma, beta, w1, b1, w2, b2)
        self.save = save
        self.norm = norm_desc(tokens, d, dtype, center, eps)
        self.up = linear_desc(tokens, f, d, dtype, act)
        self.down = linear_desc(tokens, d, f, dtype)

        def rows(cols):
            return torch.empty((tokens, cols), dtype=dt, device=dev)

        def kept(cols):
            return checkpoint_buffers(tokens, cols, dev) if save == "codes" else None

        self.h, self.u = rows(d), rows(f)
        self.mean, self.rstd = (torch.empty((tokens,), dtype=torch.float32, device=dev) for _ in range(2))
        self.x_ckpt, self.h_ckpt, self.u_ckpt = kept(d), kept(d), kept(f)
        self.z = kept(f) if save == "codes" else rows(f) if save == "rows" else None
        self.x, self.ran = None, False
        need = max(L.fs_linear_workspace(self.up, L.FS_OP_LINEAR),
                   L.fs_linear_workspace(self.down, L.FS_OP_LINEAR))
        if save:
            # (with rows saved, the backward pass still reads h and u)
            self.dh, self.du = (self.h, self.u) if save == "codes" else (rows(d), rows(f))
            need = max(need, L.fs_layer_norm_workspace(self.norm),
                       L.fs_linear_workspace(self.up, L.FS_OP_LINEAR_BACKWARD),
                       L.fs_linear_workspace(self.down, L.FS_OP_LINEAR_BACKWARD))
        self.ws = torch.empty((max(need, 256),), dtype=torch.uint8, device=dev)

    def forward(self, x, out, stream=None):
        """out = x + sublayer(x); out may be x itself, but not with
        save="rows", where the backward pass reads x, which has to stay as it
        is until then."""
        if self.save == "rows" and self.norm.rows and L.ptr(out) == L.ptr(x):
            raise ValueError("out may not be x with save='rows': the backward pass reads x")
        gamma, beta, w1, b1, w2, b2 = self.params
        self.x, self.ran = x if self.save == "rows" else None, False
        L.fs_layer_norm(self.norm, x, None, gamma, beta, None, self.h, self.mean, self.rstd,
                        save_in=self.x_ckpt, save_y=self.h_ckpt, stream=stream)
        L.fs_linear(self.up, self.h, w1, b1, None, self.u, self.ws, save_z=self.z, save_out=self.u_ckpt,
                    stream=stream)
        L.fs_linear(self.down, self.u, w2, b2, x, out, self.ws, stream=stream)
        self.ran = True
        return out

    def backward(self, dout, grads, stream=None):
        """Gradients of the last forward from dout: ``grads`` is a dict of the
        outputs "x" [tokens, d], "w1", "w2" (the parameters' type) and "gamma",
        "beta", "b1", "b2" (fp32, absent or None to leave out)."""
        if not self.save:
            raise ValueError("nothing was saved for a backward pass (save=None)")
        if not self.ran:
            raise ValueError("backward before forward")
        gamma, beta, w1, b1, w2, b2 = self.params
        x, h, u = ((self.x_ckpt, self.h_ckpt, self.u_ckpt) if self.save == "codes"
                   else (self.x, self.h, self.u))
        L.fs_linear_backward(self.down, dout, u, w2, None, self.du, grads["w2"], grads.get("b2"), self.ws,
                             stream=stream)
        L.fs_linear_backward(self.up, self.du, h, w1, self.z, self.dh, grads["w1"], grads.get("b1"),
                             self.ws, stream=stream)
        L.fs_layer_norm_backward(self.norm, self.dh, x, self.mean if self.norm.center else None, self.rstd,
                                 gamma, dout, grads["x"], grads.get("gamma"), grads.get("beta"), self.ws,
                                 stream=stream)
        return grads
