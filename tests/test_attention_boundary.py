"""Refusals of the attention sublayer's entry points, on the host before any HIP
call (no GPU needed; addresses are never dereferenced)."""

import ctypes

import pytest
import torch

import paper_2511_11505_amd as fs
from paper_2511_11505_amd import _lib as L

A, B, C, D, E, F, G = ((1 << 32) * (i + 1) for i in range(7))   # far apart, aligned, not memory
INF, NAN = float("inf"), float("nan")


def refuse(status, text, fn, *args, **kw):
    if "workspace" not in fn.__name__ and "frequencies" not in fn.__name__:
        kw["stream"] = 0
    with pytest.raises(L.FsError) as e:
        fn(*args, **kw)
    assert e.value.status == status, str(e.value)
    assert text in str(e.value), str(e.value)


def turn(first=0, rot=16, layout=0, mscale=1.0, freqs=G):
    return L.fs_rope(layout, first, rot, mscale, freqs)


def rot_desc(**kw):
    d = fs.rotary_desc(4, 2, 32)
    for f, v in kw.items():
        setattr(d, f, v)
    return d


@pytest.mark.parametrize("kw,status", [
    (dict(abi_version=1), L.FS_ERR_INVALID), (dict(dtype=2), L.FS_ERR_INVALID), (dict(tokens=-1), L.FS_ERR_INVALID),
    (dict(heads=0), L.FS_ERR_INVALID), (dict(head_dim=0), L.FS_ERR_INVALID),
    (dict(tokens=2 ** 24 + 1), L.FS_ERR_UNSUPPORTED), (dict(heads=2 ** 16 + 1), L.FS_ERR_UNSUPPORTED),
    (dict(head_dim=513), L.FS_ERR_UNSUPPORTED)])
@pytest.mark.parametrize("fn", [fs.fs_rotary, fs.fs_rotary_backward])
def test_rotary_descriptor(fn, kw, status):
    refuse(status, "", fn, rot_desc(**kw), turn(), A, B, C)


@pytest.mark.parametrize("rope", [turn(layout=2), turn(layout=-1), turn(rot=15), turn(rot=-2), turn(first=-1),
                                  turn(first=17), turn(first=33), turn(rot=34), turn(first=2 ** 31 - 1), turn(mscale=NAN),
                                  turn(mscale=INF), turn(freqs=None), turn(freqs=G + 4)])
def test_rope(rope):
    refuse(L.FS_ERR_INVALID, "rope", fs.fs_rotary, rot_desc(), rope, A, B, C)
    refuse(L.FS_ERR_INVALID, "rope", fs.fs_cache_append, cache(), rope, None, _Tokens(B), C, None, D, pages(), None)


def test_rotary_arguments():
    d = rot_desc()
    for fn, x, o in ((fs.fs_rotary, "x", "out"), (fs.fs_rotary_backward, "dout", "dx")):
        refuse(L.FS_ERR_INVALID, f"{x} must not be NULL", fn, d, turn(), None, B, C)
        refuse(L.FS_ERR_INVALID, f"{o} must not be NULL", fn, d, turn(), A, B, None)
        refuse(L.FS_ERR_INVALID, "positions", fn, d, turn(), A, None, C)
        refuse(L.FS_ERR_INVALID, "positions", fn, d, turn(), A, B + 2, C)
        refuse(L.FS_ERR_INVALID, "aligned", fn, d, turn(), A + 1, B, C)
        refuse(L.FS_ERR_INVALID, "overlap", fn, d, turn(), A, B, A + 2)
        refuse(L.FS_ERR_INVALID, "overlap", fn, d, turn(), A, B, A + 4 * 2 * 32 * 2 - 2)
        refuse(L.FS_ERR_INVALID, "overlap", fn, d, turn(), A, C + 8, C)
        refuse(L.FS_ERR_INVALID, "overlap", fn, d, turn(freqs=C + 8), A, B, C)
        fn(rot_desc(tokens=0), turn(), None, None, None, stream=0)


def test_rotary_strides():
    """Heads or tokens that overlap, and views in one another's gaps."""
    lib, d = L.load(), rot_desc()

    def call(ts, hs, x=A, out=C, tso=64, hso=32):
        return lib.fs_rotary(d, turn(), x, ts, hs, B, out, tso, hso, None)

    for ts, hs in ((0, 32), (63, 32), (64, 31), (64, 0), (-64, 32), (32, 96), (64, 64)):
        assert call(ts, hs) != L.FS_OK, (ts, hs)
        assert call(64, 32, tso=ts, hso=hs) != L.FS_OK, (ts, hs)
    assert call(64, 32, tso=1 << 41) == L.FS_ERR_UNSUPPORTED
    # the same base with other strides, and parts of one row: the output's heads
    # start inside of the input's
    assert call(128, 32, out=A, tso=64) == L.FS_ERR_INVALID
    assert call(128, 32, out=A + 2 * 48, tso=128) == L.FS_ERR_INVALID
    assert call(128, 32, out=A + 2 * (128 - 16), tso=128) == L.FS_ERR_INVALID


@pytest.mark.parametrize("args,status", [
    ((-2,), L.FS_ERR_INVALID), ((7,), L.FS_ERR_INVALID), ((514,), L.FS_ERR_UNSUPPORTED), ((8, 0.0), L.FS_ERR_INVALID),
    ((8, -1.0), L.FS_ERR_INVALID), ((8, NAN), L.FS_ERR_INVALID), ((8, INF), L.FS_ERR_INVALID),
    ((8, 1e4, "linear", 0.0), L.FS_ERR_INVALID), ((8, 1e4, "base", NAN), L.FS_ERR_INVALID),
    ((2, 1e4, "base", 2.0), L.FS_ERR_INVALID), ((8, 1e4, "parts", 2.0, 0.0), L.FS_ERR_INVALID),
    ((8, 1e4, "parts", 2.0, 64.0, 4.0, 4.0), L.FS_ERR_INVALID), ((8, 1e4, "parts", 2.0, 64.0, NAN, 4.0), L.FS_ERR_INVALID),
    ((8, 1e4, "parts", 2.0, INF, 1.0, 4.0), L.FS_ERR_INVALID)])
def test_frequencies(args, status):
    refuse(status, "", fs.fs_rope_frequencies, *args)
    assert fs.fs_rope_frequencies(0).numel() == 0
    lib = L.load()
    assert lib.fs_rope_frequencies(8, 1e4, 4, 1.0, 0.0, 0.0, 1.0, A) == L.FS_ERR_INVALID
    assert lib.fs_rope_frequencies(8, 1e4, 0, 1.0, 0.0, 0.0, 1.0, None) == L.FS_ERR_INVALID


def cache(codes=0, **kw):
    c = L.fs_kv_cache(L.FS_ABI_VERSION, L.FS_BF16, codes, 10, 2, 16, 32, 1 << 40, 2 << 40, 1024, 512, 32,
                      3 << 40 if codes else None, 4 << 40 if codes else None)
    for f, v in kw.items():
        setattr(c, f, v)
    return c


def pages(**kw):
    t = L.fs_page_table(F, 5, 3, 5)
    for f, v in kw.items():
        setattr(t, f, v)
    return t


BAD_CACHE = [
    (dict(abi_version=8), L.FS_ERR_INVALID), (dict(dtype=2), L.FS_ERR_INVALID), (dict(codes=2), L.FS_ERR_INVALID),
    (dict(n_pages=-1), L.FS_ERR_INVALID), (dict(kv_heads=0), L.FS_ERR_INVALID), (dict(page_size=0), L.FS_ERR_INVALID),
    (dict(head_dim=0), L.FS_ERR_INVALID), (dict(head_dim=36), L.FS_ERR_UNSUPPORTED),
    (dict(head_dim=264), L.FS_ERR_UNSUPPORTED), (dict(kv_heads=5000), L.FS_ERR_UNSUPPORTED),
    (dict(n_pages=2 ** 31 - 1), L.FS_ERR_UNSUPPORTED), (dict(k=None), L.FS_ERR_INVALID), (dict(v=None), L.FS_ERR_INVALID),
    (dict(k=(1 << 40) + 8), L.FS_ERR_INVALID), (dict(v=1 << 40), L.FS_ERR_INVALID), (dict(v=(1 << 40) + 64), L.FS_ERR_INVALID),
    (dict(place_stride=36), L.FS_ERR_INVALID), (dict(place_stride=24), L.FS_ERR_INVALID),
    (dict(head_stride=504), L.FS_ERR_INVALID), (dict(page_stride=1016), L.FS_ERR_INVALID),
    (dict(place_stride=1 << 21, head_stride=1 << 25, page_stride=1 << 26), L.FS_ERR_UNSUPPORTED),
    (dict(page_stride=1 << 41), L.FS_ERR_UNSUPPORTED)]


def attn(heads=4, **kw):
    d = fs.attention_desc(heads)
    for f, v in kw.items():
        setattr(d, f, v)
    return d


WS = (5 << 40, 1 << 38)


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_cache(kw, status):
    refuse(status, "", fs.fs_cache_append, cache(**kw), None, None, _heads(kw), _heads(kw, 1), None, D, pages(), None)
    refuse(status, "", fs.fs_paged_attention, attn(), cache(**kw), A, B, pages(), C, WS)


class _Tokens(int):
    """An address that also tells the binding how many tokens there are."""
    shape = (3,)


def _heads(kw, i=0):
    return _Tokens((B, C)[i])


def test_codes_need_scales():
    for kw in (dict(k_scales=None), dict(v_scales=None), dict(v_scales=3 << 40), dict(k=(1 << 40) + 4), dict(k_scales=(3 << 40) + 4),
               dict(v_scales=(4 << 40) + 1)):
        refuse(L.FS_ERR_INVALID, "", fs.fs_paged_attention, attn(), cache(1, **kw), A, B, pages(), C, WS)


@pytest.mark.parametrize("kw,status", [
    (dict(sequences=-1), L.FS_ERR_INVALID), (dict(max_pages=-1), L.FS_ERR_INVALID), (dict(ldt=4), L.FS_ERR_INVALID),
    (dict(table=None), L.FS_ERR_INVALID), (dict(table=F + 2), L.FS_ERR_INVALID),
    (dict(sequences=2 ** 20 + 1), L.FS_ERR_UNSUPPORTED), (dict(max_pages=2 ** 27, ldt=2 ** 27), L.FS_ERR_UNSUPPORTED)])
def test_pages(kw, status):
    refuse(status, "pages", fs.fs_paged_attention, attn(), cache(), A, B, pages(**kw), C, WS)
    refuse(status, "pages", fs.fs_cache_append, cache(), None, None, _Tokens(B), C, None, D, pages(**kw), None)


def test_append_arguments():
    c, t, p = cache(), _Tokens, pages()
    ap = fs.fs_cache_append
    refuse(L.FS_ERR_INVALID, "k must not be NULL", _append_c, c, k=None)
    refuse(L.FS_ERR_INVALID, "k must be", ap, c, None, None, None, C, None, D, p, None)
    refuse(L.FS_ERR_INVALID, "v must not be NULL", ap, c, None, None, t(B), None, None, D, p, None)
    refuse(L.FS_ERR_INVALID, "positions", ap, c, None, None, t(B), C, None, None, p, None)
    refuse(L.FS_ERR_INVALID, "seqs", ap, c, None, None, t(B), C, D + 2, D, p, None)
    refuse(L.FS_ERR_INVALID, "pages", ap, c, None, None, t(B), C, None, D, None, None)
    refuse(L.FS_ERR_INVALID, "cache", ap, L.fs_kv_cache(), None, None, t(B), C, None, D, p, None)
    # q and q_out go together, with heads
    for kw in (dict(q=A, out=None), dict(q=None, out=A), dict(q=A, out=E, heads=0), dict(q=A, out=E, heads=2 ** 17)):
        refuse(L.FS_ERR_INVALID, "q", _append_c, c, **kw)
    refuse(L.FS_ERR_INVALID, "tokens", _append_c, c, tokens=-1)
    refuse(L.FS_ERR_UNSUPPORTED, "tokens", _append_c, c, tokens=2 ** 24 + 1)
    # q_out apart from everything, the cache from what is read
    for other in (A, A + 2, B + 64, C, D, F, 1 << 40, (2 << 40) + 512):
        refuse(L.FS_ERR_INVALID, "overlap", _append_c, c, q=A, out=other)
    refuse(L.FS_ERR_INVALID, "overlap", _append_c, c, k=1 << 40)
    refuse(L.FS_ERR_INVALID, "overlap", _append_c, c, positions=(2 << 40) + 64)
    _append_c(c, tokens=0, k=None)


def _append_c(c, q=None, k=B, v=C, positions=D, out=None, heads=4, tokens=3, stream=0):
    L._check(L.load().fs_cache_append(c, None, tokens, heads, q, heads * 32, 32, k, 64, 32, v, 64, 32, None, positions,
                                      pages(), out, heads * 32, 32, None))


@pytest.mark.parametrize("kw,status", [
    (dict(abi_version=8), L.FS_ERR_INVALID), (dict(q_heads=0), L.FS_ERR_INVALID), (dict(q_heads=3), L.FS_ERR_INVALID),
    (dict(q_heads=2 ** 16 + 2), L.FS_ERR_UNSUPPORTED), (dict(new_tokens=0), L.FS_ERR_INVALID),
    (dict(new_tokens=2 ** 24), L.FS_ERR_UNSUPPORTED), (dict(window=-1), L.FS_ERR_INVALID),
    (dict(scale=NAN), L.FS_ERR_INVALID), (dict(scale=INF), L.FS_ERR_INVALID), (dict(scale=-3e38), L.FS_ERR_INVALID)])
def test_attention_descriptor(kw, status):
    refuse(status, "", fs.fs_paged_attention, attn(**kw), cache(), A, B, pages(), C, WS)
    refuse(status, "", fs.fs_paged_attention_workspace, attn(**kw), cache(), pages())


def test_attention_arguments():
    at, d, c, p = fs.fs_paged_attention, attn(), cache(), pages()
    refuse(L.FS_ERR_INVALID, "q must not be NULL", at, d, c, None, B, p, C, WS)
    refuse(L.FS_ERR_INVALID, "out must not be NULL", at, d, c, A, B, p, None, WS)
    refuse(L.FS_ERR_INVALID, "lengths", at, d, c, A, None, p, C, WS)
    refuse(L.FS_ERR_INVALID, "lse", at, d, c, A, B, p, C, WS, lse=D + 2)
    refuse(L.FS_ERR_INVALID, "aligned", at, d, c, A + 1, B, p, C, WS)
    long = pages(max_pages=1000, ldt=1000)
    need = fs.fs_paged_attention_workspace(d, c, long)
    assert need > 0 and fs.fs_paged_attention_workspace(d, c, pages(max_pages=2)) == 0
    refuse(L.FS_ERR_WORKSPACE, "workspace", at, d, c, A, B, long, C, (D, need - 1))
    refuse(L.FS_ERR_INVALID, "ws must", at, d, c, A, B, long, C, (D + 8, need))
    for kw in (dict(out=A), dict(out=B), dict(out=F), dict(out=1 << 40), dict(out=(2 << 40) + 2), dict(ws=(A, need)),
               dict(ws=(B, need)), dict(ws=(C, need)), dict(ws=(F, need)), dict(ws=(1 << 40, need)), dict(lse=A),
               dict(lse=C), dict(lse=WS[0])):
        a = dict(dict(out=C, ws=WS, lse=None), **kw)
        refuse(L.FS_ERR_INVALID, "overlap", at, d, c, A, B, long, a["out"], a["ws"], lse=a["lse"])
    at(d, c, None, None, pages(sequences=0), None, None, stream=0)


def test_cache_views():
    """Keys and values beside one another in a page or in a place; strides that no
    second element has are not looked at.  (The workspace is refused last.)"""
    views = [dict(k=1 << 40, v=(1 << 40) + 2 * 1024, page_stride=2048),
             dict(k=1 << 40, v=(1 << 40) + 2 * 64, page_stride=2048, place_stride=128, head_stride=32),
             dict(n_pages=1, page_stride=3), dict(kv_heads=1, head_stride=-1, page_stride=512),
             dict(page_size=1, place_stride=1 << 50, head_stride=32, page_stride=64)]
    for kw in views:
        heads = kw.get("kv_heads", 2) * 2
        refuse(L.FS_ERR_WORKSPACE, "", fs.fs_paged_attention, attn(heads), cache(**kw), A, B,
               pages(max_pages=1 << 16, ldt=1 << 16), C, (D, 0))
    # beside one another, but too near
    for kw in (dict(views[0], v=(1 << 40) + 2 * 1016), dict(views[0], v=(1 << 40) + 2 * 1032), dict(views[1], page_stride=1976)):
        refuse(L.FS_ERR_INVALID, "overlap", fs.fs_paged_attention, attn(), cache(**kw), A, B, pages(), C, WS)


def test_many_rows():
    """More workgroups than a grid holds are refused, large calls are not."""
    c = cache(kv_heads=2)
    refuse(L.FS_ERR_UNSUPPORTED, "groups of 16 rows", fs.fs_paged_attention_workspace, attn(2 ** 16, new_tokens=2 ** 11), c,
           pages(sequences=2))
    assert fs.fs_paged_attention_workspace(attn(4, new_tokens=2 ** 20), c, pages(sequences=1)) == 0
    refuse(L.FS_ERR_UNSUPPORTED, "groups of 16 rows", fs.fs_paged_attention_workspace, attn(2 ** 16, new_tokens=2 ** 24), c,
           pages(sequences=0))


def test_binding_checks():
    """Types, shapes, strides and devices of tensors (here: not on a GPU)."""
    d = rot_desc()
    x = torch.zeros((4, 2, 32), dtype=torch.bfloat16)
    pos = torch.zeros((4,), dtype=torch.int32)
    refuse(L.FS_ERR_INVALID, "current GPU", fs.fs_rotary, d, turn(), x, B, C)
    refuse(L.FS_ERR_INVALID, "current GPU", fs.fs_rotary, d, turn(), A, pos, C)
    refuse(L.FS_ERR_INVALID, "unit column stride", fs.fs_rotary, d, turn(), x.transpose(0, 2).contiguous().transpose(0, 2), B, C)
    refuse(L.FS_ERR_INVALID, "x must be", fs.fs_rotary, d, turn(), x.float(), B, C)
    refuse(L.FS_ERR_INVALID, "x must be", fs.fs_rotary, d, turn(), x[:3], B, C)
    refuse(L.FS_ERR_INVALID, "positions must be", fs.fs_rotary, d, turn(), A, pos.long(), C)
    refuse(L.FS_ERR_INVALID, "positions must be", fs.fs_rotary, d, turn(), A, torch.zeros((8,), dtype=torch.int32)[::2], C)
    f = torch.zeros((8,), dtype=torch.float64)
    refuse(L.FS_ERR_INVALID, "rope must be", fs.fs_rotary, d, fs.rope(f), A, B, C)
    with pytest.raises(L.FsError):
        fs.rope(f.float())
    with pytest.raises(ValueError):
        fs.rope(f, layout="both")
    with pytest.raises(ValueError):
        fs.fs_rope_frequencies(8, scaling="other")
    k = torch.zeros((2, 3, 4, 8), dtype=torch.bfloat16)
    s = torch.zeros((2, 3, 4, 1), dtype=torch.uint8)
    for args, kw in (((k, k.float()), {}), ((k, k[:1]), {}), ((k, k.transpose(1, 2).contiguous().transpose(1, 2)), {}),
                     ((k, k), dict(dtype="f32")), ((k, k, s, s), {}), ((k.byte(), k.byte(), s, s[..., :0]), {}),
                     ((k.byte(), k.byte(), s, None), {})):
        if kw or args[1].shape != k.shape or args[1].stride() != k.stride() or len(args) > 2 and args[0] is k:
            with pytest.raises(L.FsError):
                fs.kv_cache(*args, **kw)
    c = fs.kv_cache(k.byte(), k.byte().clone(), s, s.clone(), dtype="f32")
    assert (c.dtype, c.codes, c.n_pages, c.kv_heads, c.page_size, c.head_dim) == (L.FS_F32, 1, 2, 3, 4, 8)
    refuse(L.FS_ERR_INVALID, "cache must be", fs.fs_paged_attention, attn(3), c, A, B, pages(), C, WS)
    for t in (torch.zeros((3, 5)), torch.zeros((3,), dtype=torch.int32), torch.zeros((5, 3), dtype=torch.int32).t()):
        refuse(L.FS_ERR_INVALID, "pages must be", fs.fs_paged_attention, attn(), cache(), A, B, t, C, WS)
    refuse(L.FS_ERR_INVALID, "current GPU", fs.fs_paged_attention, attn(), cache(), A, B,
           torch.zeros((3, 5), dtype=torch.int32), C, WS)


def test_sublayer_shapes():
    c = cache()
    w = torch.zeros(((4 + 4) * 32, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        fs.AttentionSublayer(3, c, 5, None, None, w[:-1], None, w, None)
    with pytest.raises(ValueError):
        fs.AttentionSublayer(3, c, 5, None, None, w[:5 * 32], None, w, None)
    with pytest.raises(ValueError):
        fs.AttentionSublayer(3, c, 5, None, None, w, None, w, None)
    with pytest.raises(ValueError):
        fs.AttentionSublayer(3, c, 5, None, None, w.float(), None, torch.zeros((64, 128)), None)
    s = fs.AttentionSublayer(3, c, 5, None, None, w, None, torch.zeros((64, 128), dtype=torch.bfloat16), None)
    assert s.desc.q_heads == 4 and ctypes.sizeof(s.desc) == 20


def test_sizes_of_structs():
    """As the header lays them out."""
    assert [ctypes.sizeof(t) for t in (L.fs_rope, L.fs_rotary_desc, L.fs_kv_cache, L.fs_page_table,
                                       L.fs_attention_desc)] == [32, 20, 88, 24, 20]


def test_attention_at_arguments():
    """Positions are given, aligned, and apart from what is written."""
    at, d, c, p = fs.fs_paged_attention_at, attn(), cache(), pages()
    refuse(L.FS_ERR_INVALID, "positions must not be NULL", at, d, c, A, None, B, p, C, WS)
    refuse(L.FS_ERR_INVALID, "positions", at, d, c, A, D + 2, B, p, C, WS)
    refuse(L.FS_ERR_INVALID, "lengths", at, d, c, A, D, None, p, C, WS)
    refuse(L.FS_ERR_INVALID, "positions must be", at, d, c, A, torch.zeros((3,)), B, p, C, WS)
    refuse(L.FS_ERR_INVALID, "positions must be", at, attn(new_tokens=2), c, A, torch.zeros((3,), dtype=torch.int32), B, p, C, WS)
    refuse(L.FS_ERR_INVALID, "overlap", at, d, c, A, C + 8, B, p, C, WS)
    refuse(L.FS_ERR_INVALID, "overlap", at, d, c, A, D, B, p, C, WS, lse=D + 4)
    long = pages(max_pages=1000, ldt=1000)
    need = fs.fs_paged_attention_workspace(d, c, long)
    refuse(L.FS_ERR_INVALID, "overlap", at, d, c, A, D, B, long, C, (D - 256, need))
    refuse(L.FS_ERR_WORKSPACE, "workspace", at, d, c, A, D, B, long, C, (E, need - 1))
    at(d, c, None, None, None, pages(sequences=0), None, None, stream=0)


def test_kv_cache_refusals():
    """Types, shapes and strides that do not go together, and scales of one half."""
    k = torch.zeros((2, 3, 4, 8), dtype=torch.bfloat16)
    s, c = torch.zeros((2, 3, 4, 1), dtype=torch.uint8), torch.zeros((2, 3, 4, 8), dtype=torch.uint8)
    for args in ((k, k.float()), (k.float(), k), (k, k[:1]), (k, k.transpose(1, 2).contiguous().transpose(1, 2)),
                 (k, k, s, s), (k, k, s, None), (k, k, None, s), (c, c, s, s[..., :0]), (c, c, s[:1], s), (c, c, s, None),
                 (c, c, None, s), (c, c), (c, k, s, s), (c, c, s, s.int())):
        with pytest.raises(L.FsError):
            fs.kv_cache(*args)
    with pytest.raises(L.FsError):
        fs.kv_cache(k, k, dtype="f32")


def test_attention_needs_pages():
    """Without a page table: a refusal that says so, from each entry."""
    d, c = attn(), cache()
    refuse(L.FS_ERR_INVALID, "pages must", fs.fs_paged_attention, d, c, A, B, None, C, WS)
    refuse(L.FS_ERR_INVALID, "pages must", fs.fs_paged_attention_at, d, c, A, D, B, None, C, WS)
    refuse(L.FS_ERR_INVALID, "pages must", fs.fs_paged_attention_workspace, d, c, None)
    x = torch.zeros((3, 4, 32), dtype=torch.bfloat16)
    refuse(L.FS_ERR_INVALID, "pages must", fs.fs_paged_attention, d, c, x, B, None, x, None)


@pytest.mark.parametrize("codes,dtype", [(0, L.FS_BF16), (1, L.FS_BF16), (0, L.FS_F32), (1, L.FS_F32)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_workspace_of_narrower_tables(d, codes, dtype):
    """A workspace for a page table is enough for each narrower one."""
    c = cache(codes, head_dim=d, dtype=dtype, place_stride=d, head_stride=16 * d, page_stride=32 * d, page_size=16)
    for rows in (1, 8, 17, 32, 33, 64, 65, 200):
        for sequences in (1, 3, 40, 700, 3000):
            most = 0
            for n in sorted({2 ** i + j for i in range(14) for j in (-1, 0, 1)} | {11000}):
                p = pages(max_pages=n, ldt=n, sequences=sequences)
                need = fs.fs_paged_attention_workspace(attn(2 * rows), c, p)
                assert need >= most, (rows, sequences, n, need, most)
                most = need
