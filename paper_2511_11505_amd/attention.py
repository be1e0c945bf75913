"""The attention sublayer of a serving step that runs in the far-skip window.

FarSkip runs the next layer's attention between the block's BEGIN and FINISH
phases, on an input that lacks the block's routed output (Section 3, Eq. 8b;
the split of Section 4.1).  ``AttentionSublayer`` is that computation for the new
tokens of a batch of sequences, over their paged key-value cache:

    h = norm(x);  q, k, v = h w_qkv^T + b_qkv;  k and v appended, q and k turned
    out = x + attention(q, cache) w_out^T + b_out

through fs_layer_norm, fs_linear, fs_cache_append and fs_paged_attention_at.  All
arithmetic runs in the library's kernels; torch only allocates memory.  A
sublayer's passes share its buffers and its workspace, so they run one after
another, on one stream or ordered by events.
"""

import torch

from . import _lib as L
from .sublayer import _TYPES, linear_desc, norm_desc


def empty_cache(pages, page_size, kv_heads, head_dim, dtype="bf16", codes=False, device="cuda"):
    """fs_kv_cache of uninitialised memory: rows of dtype, or with ``codes`` 8-bit
    codes and their scales.  Its tensors are in ``.tensors`` (k, v, k_scales,
    v_scales)."""
    shape = (pages, kv_heads, page_size, head_dim)
    kind = torch.uint8 if codes else _TYPES[dtype][1]
    k, v = (torch.empty(shape, dtype=kind, device=device) for _ in range(2))
    if not codes:
        return L.kv_cache(k, v, dtype=dtype)
    scales = (torch.empty((*shape[:3], (head_dim + 31) // 32), dtype=torch.uint8, device=device) for _ in range(2))
    return L.kv_cache(k, v, *scales, dtype=dtype)


class AttentionSublayer:
    def __init__(self, sequences, cache, max_pages, gamma, beta, w_qkv, b_qkv, w_out, b_out, rope=None,
                 new_tokens=1, center=False, eps=1e-5, scale=None, window=0):
        """gamma, beta [d] fp32 or None; w_qkv [(heads + 2 kv_heads) head_dim, d],
        w_out [d, heads head_dim] of the cache's dtype; b_qkv, b_out fp32 or None.
        Each pass is of sequences * new_tokens tokens; max_pages: the page table's
        columns."""
        (n, d), hd, kv = w_qkv.shape, cache.head_dim, cache.kv_heads
        heads = n // hd - 2 * kv
        if n % hd or heads < kv or heads % kv:
            raise ValueError(f"w_qkv must be [(heads + {2 * kv}) * {hd}, d] with heads a multiple of {kv}, "
                             f"not {list(w_qkv.shape)}")
        if tuple(w_out.shape) != (d, heads * hd):
            raise ValueError(f"w_out must be [{d}, {heads * hd}], not {list(w_out.shape)}")
        dtype = "f32" if cache.dtype == L.FS_F32 else "bf16"
        dt, dev = _TYPES[dtype][1], w_qkv.device
        if w_qkv.dtype != dt or w_out.dtype != dt:
            raise ValueError(f"w_qkv and w_out must be {dt}, the cache's dtype")
        tokens = sequences * new_tokens
        self.params, self.cache, self.rope = (gamma, beta, w_qkv, b_qkv, w_out, b_out), cache, rope
        self.norm = norm_desc(tokens, d, dtype, center, eps)
        self.qkv_desc = linear_desc(tokens, n, d, dtype)
        self.out_desc = linear_desc(tokens, d, heads * hd, dtype)
        self.desc = L.attention_desc(heads, new_tokens, hd ** -0.5 if scale is None else scale, window)

        def rows(cols):
            return torch.empty((tokens, cols), dtype=dt, device=dev)

        self.h, self.qkv, self.q, self.o = rows(d), rows(n), rows(heads * hd), rows(heads * hd)
        self.heads = tuple(t.view(tokens, -1, hd) for t in (self.qkv, self.q, self.o))
        self.mean, self.rstd = (torch.empty((tokens,), dtype=torch.float32, device=dev) for _ in range(2))
        self.seqs = None if new_tokens == 1 else torch.arange(
            sequences, dtype=torch.int32, device=dev).repeat_interleave(new_tokens)
        need = max(L.fs_linear_workspace(self.qkv_desc, L.FS_OP_LINEAR),
                   L.fs_linear_workspace(self.out_desc, L.FS_OP_LINEAR),
                   L.fs_paged_attention_workspace(self.desc, cache, L.fs_page_table(None, max_pages, sequences,
                                                                                     max_pages)))
        self.ws = torch.empty((max(need, 256),), dtype=torch.uint8, device=dev)

    def forward(self, x, out, positions, lengths, pages, stream=None):
        """out [tokens, d] = x + sublayer(x); out may be x itself.  Token i of
        sequence b is row b * new_tokens + i; positions [tokens] int32: its place
        in the sequence (negative: none, as a padded batch has them first or last);
        lengths [sequences] int32: tokens that the sequence has with the new ones;
        pages [sequences, max_pages] int32.  Of a token that is none the attention
        is 0."""
        gamma, beta, w_qkv, b_qkv, w_out, b_out = self.params
        qkv, q, o = self.heads
        h, kv = self.desc.q_heads, self.cache.kv_heads
        L.fs_layer_norm(self.norm, x, None, gamma, beta, None, self.h, self.mean, self.rstd, stream=stream)
        L.fs_linear(self.qkv_desc, self.h, w_qkv, b_qkv, None, self.qkv, self.ws, stream=stream)
        L.fs_cache_append(self.cache, self.rope, qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:], self.seqs, positions,
                          pages, q, stream=stream)
        L.fs_paged_attention_at(self.desc, self.cache, q, positions, lengths, pages, o, self.ws, stream=stream)
        L.fs_linear(self.out_desc, self.o, w_out, b_out, x, out, self.ws, stream=stream)
        return out
