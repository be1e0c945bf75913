"""Rotary positions, the append to a paged cache and paged attention on the GPU
against the fp64 oracle.

Tolerances are bounds, from the operations that round (2^-24 each in fp32, half a
step of a stored type: bf16 2^-8 of the value, fp32 2^-24).

Rotation: cos, sin, each product and the sum round once: 3 * 2^-24 of
mscale (|a| + |b|), then the store.

Attention: a score of d products errs by at most (d + 2) 2^-23 of sum |q k| scale
(products and adds, and the factor scale log2 e with its own rounding); the
exponential turns that into a relative error, and its own is at most 2^-21; a sum
of L weights errs by L 2^-24 of it, the rescalings (at most one for each of 64 first
tiles and each join) by 2^-20; a weight that is rounded to bf16 by 2^-8, one that is
kept as two bf16 numbers by 2^-16 (a bf16 cache with at most 32 rows a key head).  An output
errs by that much of sum |weight v|, twice (sum of values, sum of weights), then
the store."""

import numpy as np
import pytest
import torch

import paper_2511_11505_amd as fs
from oracle import attention as O
from paper_2511_11505_amd import _lib as L
from tests._util import f64

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]
DEV = "cuda"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
U = 2.0 ** -23


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def heads(g, tokens, n, d, dtype, pad=0, lead=0, head_major=False, scale=1.0):
    """[tokens, n, d] view inside NaNs."""
    a, b = (n, tokens) if head_major else (tokens, n)
    full = torch.full((a * (b * d + pad) + pad + lead + 64,), float("nan"), dtype=TORCH[dtype], device=DEV)
    v = full[lead:lead + a * (b * d + pad)].view(a, b * d + pad)[:, :b * d].unflatten(1, (b, d))
    v = v.transpose(0, 1) if head_major else v
    v.copy_(scale * torch.randn((tokens, n, d), generator=g, device=DEV))
    return v


class Out:
    """An output inside a buffer of a sentinel, which has to stay."""

    def __init__(self, tokens, n, d, dtype, pad=0, lead=0):
        self.full = torch.full((tokens * (n * d + pad) + lead + 64,), -77.0, dtype=TORCH[dtype], device=DEV)
        self.at = (tokens, n, d, pad, lead)
        self.view = self.cut(self.full)

    def cut(self, full):
        tokens, n, d, pad, lead = self.at
        return full[lead:lead + tokens * (n * d + pad)].view(tokens, n * d + pad)[:, :n * d].unflatten(1, (n, d))

    def get(self):
        rest = self.full.clone()
        self.cut(rest).fill_(-77.0)
        assert bool((rest == -77.0).all()), "wrote outside the output"
        return f64(self.view)


def near(got, want, tol):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4],
                           np.broadcast_to(tol, got.shape)[bad][:4])


def turn_tol(x, freqs, layout, first, mscale, want, dtype):
    a, b = O.pairs(2 * len(freqs), layout, first)
    size = np.zeros(x.shape)
    both = np.abs(x[..., a]) + np.abs(x[..., b])
    size[..., a], size[..., b] = both, both
    t = 3 * 2.0 ** -24 * abs(mscale) * size
    return t + HALF[dtype] * (np.abs(want) + t)


def spun(rot, layout, first=0, mscale=1.0, **kw):
    f = fs.fs_rope_frequencies(rot, **kw)
    return f.numpy(), fs.rope(f.to(DEV), layout=layout, first=first, mscale=mscale)


# ------------------------------------------------------------------- rotary
ROTARY = [  # tokens, heads, d, rot, first, pad, lead
    (1, 1, 2, 2, 0, 0, 0), (1, 48, 128, 128, 0, 0, 0), (3, 5, 64, 64, 0, 0, 0), (5, 3, 75, 38, 3, 5, 1),
    (257, 7, 128, 64, 64, 0, 0), (130, 9, 192, 64, 128, 8, 0), (17, 2, 256, 256, 0, 1, 0), (2, 3, 512, 512, 0, 0, 0),
    (9, 1, 511, 500, 11, 3, 1), (33, 4, 96, 20, 4, 0, 0), (1, 300, 8, 8, 0, 0, 0), (4, 6, 16, 0, 5, 0, 0),
    (700, 33, 72, 48, 16, 8, 0), (5000, 2, 24, 16, 8, 0, 0)]


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", ROTARY, ids=str)
def test_rotary(case, dtype, layout):
    tokens, n, d, rot, first, pad, lead = case
    g = gen(tokens + d)
    x = heads(g, tokens, n, d, dtype, pad, lead)
    pos = torch.randint(-50, 1 << 20, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    freqs, rope = spun(rot, layout, first, 1.25, scaling="linear", factor=2.0)
    desc = fs.rotary_desc(tokens, n, d, dtype)
    for back, call in ((False, fs.fs_rotary), (True, fs.fs_rotary_backward)):
        out = Out(tokens, n, d, dtype, pad, lead)
        call(desc, rope, x, pos, out.view)
        torch.cuda.synchronize()
        want = O.rotary(f64(x), pos.cpu().numpy(), freqs, layout, first, 1.25, back)
        near(out.get(), want, turn_tol(f64(x), freqs, layout, first, 1.25, want, dtype))
        # in place: the same bits
        y = heads(g, tokens, n, d, dtype, pad, lead)
        y.copy_(x)
        call(desc, rope, y, pos, y)
        torch.cuda.synchronize()
        assert torch.equal(y, out.view)


def test_rotary_head_major():
    """Heads that hold their tokens, and an output of the other order."""
    g = gen(3)
    x = heads(g, 65, 6, 64, "bf16", 8, head_major=True)
    pos = torch.randint(0, 5000, (65,), generator=g, device=DEV, dtype=torch.int32)
    freqs, rope = spun(32, "pairs", 16)
    out = Out(65, 6, 64, "bf16")
    fs.fs_rotary(fs.rotary_desc(65, 6, 64), rope, x, pos, out.view)
    torch.cuda.synchronize()
    want = O.rotary(f64(x), pos.cpu().numpy(), freqs, "pairs", 16)
    near(out.get(), want, turn_tol(f64(x), freqs, "pairs", 16, 1.0, want, "bf16"))


def test_rotary_far_positions():
    """The ends of the positions' range: angles are products in 64 bits."""
    pos = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 0, 1], dtype=torch.int32, device=DEV)
    x = heads(gen(5), 5, 2, 64, "f32")
    freqs, rope = spun(64, "halves")
    out = Out(5, 2, 64, "f32")
    fs.fs_rotary(fs.rotary_desc(5, 2, 64, "f32"), rope, x, pos, out.view)
    torch.cuda.synchronize()
    want = O.rotary(f64(x), pos.cpu().numpy(), freqs, "halves")
    # (angles of 2^31 radians in 64 bits: 2^-22 absolute, on both sides)
    near(out.get(), want, turn_tol(f64(x), freqs, "halves", 0, 1.0, want, "f32") + 2.0 ** -21 * np.abs(f64(x)).max())
    near(out.get()[3:], want[3:], turn_tol(f64(x), freqs, "halves", 0, 1.0, want, "f32")[3:])


def test_rotary_keeps_what_is_beside():
    """Infinities and NaNs stay in their pairs and in columns that do not turn."""
    x = torch.randn((4, 2, 64), generator=gen(1), device=DEV)
    x[0, 0, 3], x[1, 1, 60], x[2, 0, 40] = float("inf"), float("nan"), float("-inf")
    pos = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device=DEV)
    freqs, rope = spun(32, "halves")
    out = torch.empty_like(x)
    fs.fs_rotary(fs.rotary_desc(4, 2, 64, "f32"), rope, x, pos, out)
    torch.cuda.synchronize()
    bad = ~torch.isfinite(out)
    assert bad.nonzero().tolist() == [[0, 0, 3], [0, 0, 19], [1, 1, 60], [2, 0, 40]]
    assert torch.isnan(out[1, 1, 60]) and out[2, 0, 40] == float("-inf")


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_rotary_gradient_by_differences(layout):
    """<dout, f(x + h e) - f(x - h e)> / 2 h is dx . e: f is linear, so the only
    errors are roundings: of both outputs (3 * 2^-24 each), of dx and of the sums."""
    g = gen(11)
    x, dout, e = (heads(g, 6, 3, 48, "f32") for _ in range(3))
    pos = torch.randint(0, 9000, (6,), generator=g, device=DEV, dtype=torch.int32)
    _, rope = spun(32, layout, 8, 1.5)
    desc = fs.rotary_desc(6, 3, 48, "f32")
    up, down, dx = (torch.empty((6, 3, 48), device=DEV) for _ in range(3))
    fs.fs_rotary(desc, rope, x + e, pos, up)
    fs.fs_rotary(desc, rope, x - e, pos, down)
    fs.fs_rotary_backward(desc, rope, dout, pos, dx)
    torch.cuda.synchronize()
    lhs = (f64(dout) * (f64(up) - f64(down))).sum() / 2
    rhs = (f64(dx) * f64(e)).sum()
    size = (np.abs(f64(dout)).sum() + np.abs(f64(e)).sum()) * 2 * 1.5 * 4 * (
        np.abs(f64(x)).max() + np.abs(f64(e)).max() + np.abs(f64(dout)).max())
    assert abs(lhs - rhs) <= 4 * 2.0 ** -24 * size


# -------------------------------------------------------------------- cache
class Cache:
    """A cache of random values, or of NaNs, with the strides of a larger one
    whose rest is a sentinel."""

    def __init__(self, g, pages, kv, size, d, dtype, codes=False, order="heads", gap=0, poison=False):
        shape = {"heads": (pages, kv, size, d + gap), "tokens": (pages, size, kv, d + gap)}[order]
        dt = torch.uint8 if codes else TORCH[dtype]

        def make():
            full = torch.full(shape, 0x33 if codes else -77.0, dtype=dt, device=DEV)
            v = full if order == "heads" else full.transpose(1, 2)
            return full, v[..., :d]

        self.full, self.k = make()
        self.fullv, self.v = make()
        self.ks = self.vs = None
        self.d, self.codes, self.dtype = d, codes, dtype
        if codes:
            nb = (d + 31) // 32
            self.ks, self.vs = (torch.full((pages, kv, size, nb), 255 if poison else 127, dtype=torch.uint8, device=DEV)
                                for _ in range(2))
        for x, s in ((self.k, self.ks), (self.v, self.vs)):
            if poison:
                x.fill_(0x7F if codes else float("nan"))
            elif codes:
                x.copy_(torch.randint(0, 127, x.shape, generator=g, device=DEV) * 1
                        + 128 * torch.randint(0, 2, x.shape, generator=g, device=DEV))
                x.bitwise_and_(0xBF)          # (below 2^1: softmaxes of more than one token)
                s.copy_(torch.randint(124, 128, s.shape, generator=g, device=DEV))
            else:
                x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        self.struct = fs.kv_cache(self.k, self.v, self.ks, self.vs, dtype=dtype)

    def values(self):
        if self.codes:
            return tuple(O.decoded(x.contiguous().cpu().numpy(), s.cpu().numpy())
                         for x, s in ((self.k, self.ks), (self.v, self.vs)))
        return f64(self.k), f64(self.v)

    def gaps(self):
        for full in (self.full, self.fullv):
            rest = full[..., self.d:]
            assert bool((rest == (0x33 if self.codes else -77.0)).all()), "wrote between the rows"


def pages_of(g, lens, size, spare=2, width=None):
    """A table with every sequence's pages in random order; other entries bad."""
    counts = [(max(n, 0) + size - 1) // size for n in lens]
    total = sum(counts) + spare
    order = torch.randperm(total, generator=g, device=DEV).int()
    full = torch.full((len(lens), (width or max(1, *counts, 1)) + 3), 2 ** 30, dtype=torch.int32, device=DEV)
    table = full[:, :full.shape[1] - 3]
    table.fill_(-1)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    return table, total


APPEND = [  # tokens per sequence, starts, q heads, kv heads, d, rot, first, page, layout, pad
    ([1, 1, 1], [0, 17, 63], 4, 2, 128, 128, 0, 16, "halves", 0),
    ([5, 0, 40], [3, 9, 0], 6, 3, 80, 40, 16, 21, "pairs", 3),
    ([33], [31], 1, 1, 8, 8, 0, 1, "halves", 0),
    ([7, 2], [100, 0], 40, 8, 128, 64, 64, 64, "halves", 8),
    ([64, 64], [0, 5], 2, 2, 256, 256, 0, 7, "pairs", 0),
    ([9], [0], 3, 3, 72, 20, 4, 5, "halves", 1),
    ([300, 1], [10, 700], 5, 1, 64, 0, 0, 48, "halves", 0)]


@pytest.mark.parametrize("order", ["heads", "tokens"])
@pytest.mark.parametrize("kind", ["bf16", "f32", "bf16 codes", "f32 codes"])
@pytest.mark.parametrize("case", APPEND, ids=str)
def test_append(case, kind, order):
    counts, starts, h, kv, d, rot, first, size, layout, pad = case
    dtype, codes = kind.split()[0], "codes" in kind
    g = gen(d + size)
    table, pages = pages_of(g, [a + b for a, b in zip(counts, starts)], size)
    cache = Cache(g, pages, kv, size, d, dtype, codes, order, gap=8)
    before = cache.values()
    seqs = [b for b, n in enumerate(counts) for _ in range(n)]
    pos = [s + i for s, n in zip(starts, counts) for i in range(n)]
    # tokens in any order, some of them none
    perm = torch.randperm(len(seqs), generator=g, device=DEV).tolist()
    seqs, pos = [seqs[i] for i in perm] + [0, -1, len(counts)], [pos[i] for i in perm] + [-1, 3, 3]
    t = len(seqs)
    qkv = heads(g, t, h + 2 * kv, d, dtype, pad)
    q, k, v = qkv.split((h, kv, kv), dim=1)
    freqs, rope = spun(rot, layout, first, 0.75)
    out = Out(t, h, d, dtype, pad)
    fs.fs_cache_append(cache.struct, rope, q, k, v, torch.tensor(seqs, dtype=torch.int32, device=DEV),
                       torch.tensor(pos, dtype=torch.int32, device=DEV), table, out.view)
    torch.cuda.synchronize()
    cache.gaps()
    Q, K, V = f64(q), f64(k), f64(v)
    want = O.rotary(Q, pos, freqs, layout, first, 0.75)
    tol = turn_tol(Q, freqs, layout, first, 0.75, want, dtype)
    want[-3:], tol[-3:] = 0.0, 0.0
    near(out.get(), want, tol)
    turned = O.rotary(K, pos, freqs, layout, first, 0.75)
    tol = turn_tol(K, freqs, layout, first, 0.75, turned, "f32" if codes else dtype)
    got_k, got_v = cache.values()
    tb = table.cpu().numpy()
    old_k, old_v = before
    if codes:
        # half a code's step: 2^-4 of the value, of the least normal code (2^-6)
        # of the block's scale below it; a block's scale may differ by a rounding
        # of its largest value
        _, scales = O.coded(turned)
        step = 2.0 ** (np.repeat(scales.astype(float), 32, axis=-1)[..., :d] - 127)
        tol = 2 * (tol + np.maximum(2.0 ** -4 * np.abs(turned), 2.0 ** -10 * step))
        V = O.decoded(*O.coded(V))
    near(got_k, O.append(old_k, turned, seqs, pos, tb), O.append(np.zeros(old_k.shape), tol, seqs, pos, tb))
    near(got_v, O.append(old_v, V, seqs, pos, tb), 0.0)


def test_append_turned_codes_are_those_of_the_fp32_rows():
    """The codes of turned rows: an fp32 cache's rows, coded."""
    g = gen(2)
    table, pages = pages_of(g, [50], 16)
    k, v = heads(g, 50, 2, 96, "f32"), heads(g, 50, 2, 96, "f32")
    pos = torch.arange(50, dtype=torch.int32, device=DEV)
    seqs = torch.zeros_like(pos)
    _, rope = spun(96, "halves")
    rows, coded = (Cache(g, pages, 2, 16, 96, "f32", codes) for codes in (False, True))
    for c in (rows, coded):
        fs.fs_cache_append(c.struct, rope, None, k, v, seqs, pos, table, None)
    torch.cuda.synchronize()
    for x, codes, scales in ((rows.k, coded.k, coded.ks), (rows.v, coded.v, coded.vs)):
        at = [(int(table[0, p // 16]), p % 16) for p in range(50)]
        want = O.coded(np.stack([f64(x[a, :, b]) for a, b in at]))
        assert np.array_equal(want[0], np.stack([codes[a, :, b].cpu().numpy() for a, b in at]))
        assert np.array_equal(want[1], np.stack([scales[a, :, b].cpu().numpy() for a, b in at]))


def test_append_holes():
    """Bad entries of the table, positions behind it, no sequence ids, no rotation;
    infinities and NaNs as codes."""
    g = gen(9)
    table = torch.tensor([[-1, 0], [1, 7], [2 ** 31 - 1, -2 ** 31], [2, 3]], dtype=torch.int32, device=DEV)
    for codes in (False, True):
        cache = Cache(g, 4, 2, 4, 32, "bf16", codes)
        before = cache.values()
        k, v = heads(g, 4, 2, 32, "bf16"), heads(g, 4, 2, 32, "bf16")
        k[3, 1, 5], v[3, 0, 0] = float("inf"), float("nan")
        pos = torch.tensor([0, 5, 1, 6], dtype=torch.int32, device=DEV)
        fs.fs_cache_append(cache.struct, None, None, k, v, None, pos, table, None)
        fs.fs_cache_append(cache.struct, None, None, k, v, None, pos + 100, table, None)
        torch.cuda.synchronize()
        got = cache.values()
        for x, (old, new) in zip((k, v), zip(before, got)):
            changed = np.argwhere((old != new).any((1, 3)))
            assert changed.tolist() == [[3, 2]]
            want = f64(x[3])
            if codes:
                want = O.decoded(*O.coded(want))
            assert np.array_equal(new[3, :, 2], want, equal_nan=True)


# ---------------------------------------------------------------- attention
LENGTHS = {"small": [0, 1, 2, 15, 16, 17, 31, 33], "mid": [63, 64, 65, 300, 1, 0, 129, 128], "long": [1000, 3, 2049, 0],
           "one": [4097]}


def check_attention(kind, h, kv, d, lens, size, new=1, window=0, pad=0, order="heads", gap=0, seed=0, scale=None,
                    holes=(), lead=0, tokens=0):
    dtype, codes = kind.split()[0], "codes" in kind
    g = gen(seed + d + size + h)
    table, pages = pages_of(g, lens, size, width=tokens // size)
    cache = Cache(g, pages, kv, size, d, dtype, codes, order, gap, poison=True)
    real = Cache(g, pages, kv, size, d, dtype, codes, order, gap)
    # only the places that hold tokens are not NaN
    for b, n in enumerate(lens):
        for j in range(n):
            a, p = int(table[b, j // size]), j % size
            for x, y in ((cache.k, real.k), (cache.v, real.v), (cache.ks, real.ks), (cache.vs, real.vs)):
                if x is not None:
                    x[a, :, p] = y[a, :, p]
            if size >= 16 and p == 0:      # whole pages at once
                stop = min(size, n - j)
                for x, y in ((cache.k, real.k), (cache.v, real.v), (cache.ks, real.ks), (cache.vs, real.vs)):
                    if x is not None:
                        x[a, :, :stop] = y[a, :, :stop]
    for b, slot, value in holes:
        table[b, slot] = value
    t = len(lens) * new
    q = heads(g, t, h, d, dtype, pad, lead)
    scale = d ** -0.5 if scale is None else scale
    desc = fs.attention_desc(h, new, scale, window)
    need = fs.fs_paged_attention_workspace(desc, cache.struct, table)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    out = Out(t, h, d, dtype, pad, lead)
    lse = torch.full((t + 1, h), -77.0, device=DEV)
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    fs.fs_paged_attention(desc, cache.struct, q, lengths, table, out.view, (ws.data_ptr(), need), lse=lse[:t])
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0xFF).all()) and bool((lse[t] == -77.0).all())
    k, v = cache.values()
    want, want_lse, mass, reach = O.attention(f64(q), k, v, lens, table.cpu().numpy(), new, float(np.float32(scale)),
                                              window)
    got, got_lse = out.get(), f64(lse[:t])
    longest = max(lens)
    err = np.expm1((d + 2) * U * reach) + 2.0 ** -21 + longest * 2.0 ** -24 + 2.0 ** -20
    once = codes or new * h // kv > 32
    weight = err + (0 if dtype == "f32" else 2.0 ** -8 if once else 2.0 ** -16)
    tol = (2 * weight)[..., None] * mass
    near(got, want, tol + HALF[dtype] * (np.abs(want) + tol))
    none = np.isneginf(want_lse)
    assert np.array_equal(none, np.isneginf(got_lse)) and (got[none] == 0).all()
    near(got_lse[~none], want_lse[~none], (2 * err + 2.0 ** -22 * np.abs(np.where(none, 0, want_lse)))[~none])
    # the same call gives the same bits, without lse too
    again = Out(t, h, d, dtype, pad, lead)
    fs.fs_paged_attention(desc, cache.struct, q, lengths, table, again.view, (ws.data_ptr(), need))
    torch.cuda.synchronize()
    assert np.array_equal(again.get(), got)


KINDS = ["bf16", "f32", "bf16 codes", "f32 codes"]


@pytest.mark.parametrize("lens", ["small", "mid"])
@pytest.mark.parametrize("size", [1, 5, 16, 48])
@pytest.mark.parametrize("kind", KINDS)
def test_attention(kind, size, lens):
    check_attention(kind, 10, 2, 128, LENGTHS[lens], size)


@pytest.mark.parametrize("d", [8, 64, 72, 96, 136, 192, 256])
@pytest.mark.parametrize("kind", KINDS)
def test_attention_widths(kind, d):
    check_attention(kind, 3, 3, d, LENGTHS["small"], 16)
    check_attention(kind, 4, 2, d, [70, 700, 5], 20, new=2)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("h,kv,new", [(1, 1, 1), (7, 1, 1), (16, 1, 1), (17, 1, 1), (32, 1, 1), (33, 1, 1), (64, 1, 1),
                                      (65, 1, 2), (10, 5, 7), (40, 8, 4), (4, 4, 40)])
def test_attention_rows(kind, h, kv, new):
    """Query heads of a key head and new tokens, up to more rows than one tile
    holds; sequences shorter than the new tokens."""
    check_attention(kind, h, kv, 64, [90, 3, 0, 41], 16, new=new)
    check_attention(kind, h, kv, 128, [600, 20], 16, new=new)


@pytest.mark.parametrize("kind", ["bf16", "f32", "bf16 codes"])
@pytest.mark.parametrize("window", [1, 5, 16, 33, 200, 5000, 2 ** 31 - 1])
@pytest.mark.parametrize("new", [1, 3])
def test_attention_window(kind, window, new):
    check_attention(kind, 4, 2, 128, LENGTHS["mid"], 16, new=new, window=window)
    check_attention(kind, 4, 2, 64, LENGTHS["mid"], 7, new=new, window=window)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size,window", [(16, 0), (7, 0), (16, 30)])
def test_attention_prompts(kind, size, window):
    """So many new tokens that each wave has rows of its own: a sequence with tokens
    before them, one of them alone, shorter ones, an empty one."""
    lens = [150, 70, 69, 3, 0, 71, 70, 100, 12, 90, 70, 33]
    check_attention(kind, 20, 5, 64, lens, size, new=70, window=window)
    if not window:
        check_attention(kind, 20, 5, 72, lens, size, new=70)
        check_attention(kind, 20, 5, 136, lens, size, new=70)


@pytest.mark.parametrize("kind", ["bf16", "bf16 codes"])
@pytest.mark.parametrize("size,window", [(16, 0), (7, 0), (16, 30), (5, 9)])
@pytest.mark.parametrize("new,d", [(70, 64), (68, 40), (70, 128), (68, 72)])
def test_attention_prompts_of_two_tiles(kind, size, window, new, d):
    """The same with 32 rows a wave, and a last one with 24 or 16."""
    lens = [150, new, new - 1, 3, 0, new + 1, new, 100, 12, 90, 70, 33]
    check_attention(kind, 24, 6, d, lens, size, new=new, window=window)


@pytest.mark.parametrize("kind", KINDS)
def test_attention_many_rows(kind):
    """Row groups of one key head, divided and not."""
    check_attention(kind, 20, 1, 256, [400, 90], 16, new=17)
    check_attention(kind, 20, 1, 64, [90], 16, new=60)
    check_attention(kind, 300, 1, 128, [333], 16)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens", ["long", "one"])
def test_attention_divided(kind, lens):
    """Sequences in several parts, and parts of several sequences."""
    check_attention(kind, 5, 1, 128, LENGTHS[lens], 16)
    check_attention(kind, 6, 3, 72, LENGTHS[lens], 9, new=2)


@pytest.mark.parametrize("kind", ["bf16", "bf16 codes"])
@pytest.mark.parametrize("size", [16, 5])
@pytest.mark.parametrize("d", [40, 64, 128])
def test_attention_many_rows_of_a_long_table(kind, size, d):
    """Over 32 rows a key head where the table has room for 2^18 tokens and heads:
    short and long sequences, divided and not."""
    for new, lens in ((4, [900, 0, 3, 64, 2500]), (7, [31, 1, 700])):
        check_attention(kind, 33, 3, d, lens, size, new=new, tokens=40000)
        check_attention(kind, 33, 3, d, lens, size, new=new, tokens=40000, window=45)


def test_attention_many_rows_undivided():
    g = torch.Generator().manual_seed(6)
    lens = torch.randint(0, 9, (4200,), generator=g).tolist()
    lens[4100] = 650
    check_attention("bf16", 36, 1, 64, lens, 16)


@pytest.mark.parametrize("kind", ["bf16", "f32", "bf16 codes"])
def test_attention_many_sequences(kind):
    """More sequences than the scan has threads, and more than are divided."""
    g = torch.Generator().manual_seed(4)
    lens = torch.randint(0, 40, (600,), generator=g).tolist()
    lens[77] = 900
    check_attention(kind, 2, 1, 64, lens, 16)


def test_attention_many_key_heads():
    """Key heads that fill the chip alone: parts of whole sequences, and none."""
    check_attention("bf16", 300, 300, 8, [700, 30], 16)
    check_attention("f32", 520, 520, 8, [700, 30], 16)


@pytest.mark.parametrize("kind", ["bf16", "f32 codes"])
def test_attention_strides(kind):
    check_attention(kind, 6, 2, 80, [50, 130, 0], 16, order="tokens", gap=8, pad=3, lead=1)
    check_attention(kind, 6, 2, 128, [50, 300, 0], 16, order="tokens", gap=0, pad=8)


@pytest.mark.parametrize("kind", ["bf16", "f32", "bf16 codes"])
@pytest.mark.parametrize("size", [16, 5])
def test_attention_holes(kind, size):
    """Pages that are not there; a sequence without any."""
    lens = [100, 16, 40, 33]
    holes = [(0, 1, -1), (0, 3, 2 ** 31 - 1), (2, 0, -2 ** 31)] + [(1, i, 999) for i in range((16 + size - 1) // size)]
    check_attention(kind, 4, 2, 64, lens, size, holes=holes)
    check_attention(kind, 4, 2, 64, lens, size, holes=holes, new=3, window=20)


def test_attention_scales():
    """A factor of 0, a negative one, and one that leaves one token."""
    for scale in (0.0, -0.5, 40.0):
        check_attention("f32", 4, 2, 64, [5, 70, 33], 16, scale=scale)
        check_attention("bf16", 4, 2, 64, [5, 70, 33], 16, scale=scale)


# ------------------------------------------- what does not reach, and what does
def place_of(table, size, b, j):
    return int(table[b, j // size]), j % size


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [16, 5])
def test_attention_values_that_are_not_finite(kind, size):
    """An infinite or NaN value reaches the queries that see it, in its column (in
    its block of a coded cache), and no other."""
    dtype, codes = kind.split()[0], "codes" in kind
    # (the third and the last: a wave has its rows to itself; the fourth: four row
    # tiles a wave over a long table)
    for window, lens, new, tokens in ((0, [40, 9], 5, 0), (6, [40, 9], 5, 0), (0, [240, 9] + [232] * 10, 232, 0),
                                      (0, [40, 17], 15, 70000), (0, [240, 9] + [232] * 16, 232, 0)):
        g = gen(21)
        d = 64
        table, pages = pages_of(g, lens, size, width=tokens // size)
        cache = Cache(g, pages, 2, size, d, dtype, codes)
        q = heads(g, len(lens) * new, 6, d, dtype)
        desc = fs.attention_desc(6, new, d ** -0.5, window)
        ws = torch.empty((fs.fs_paged_attention_workspace(desc, cache.struct, table) + 256,), dtype=torch.uint8, device=DEV)
        lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
        bad = [(0, 38, 0, 3, float("nan")), (0, 37, 1, 40, float("inf")), (1, 8, 0, 63, float("-inf")),
               (1, 2, 1, 0, float("inf"))]
        for b, j, h, c, value in bad:
            pg, pl = place_of(table, size, b, j)
            if codes:
                cache.v[pg, h, pl, c // 32 * 32:c // 32 * 32 + 32] = 0x7F
                cache.vs[pg, h, pl, c // 32] = 255
            else:
                cache.v[pg, h, pl, c] = value
        out = Out(len(lens) * new, 6, d, dtype)
        fs.fs_paged_attention(desc, cache.struct, q, lengths, table, out.view, ws)
        torch.cuda.synchronize()
        got = out.get()
        want = np.zeros(got.shape)
        for b, j, h, c, value in bad:
            for i in range(new):
                at = lens[b] - new + i
                if j <= at and (not window or j > at - window):
                    cols = slice(c // 32 * 32, c // 32 * 32 + 32) if codes else c
                    want[b * new + i, h * 3:h * 3 + 3, cols] = np.nan if codes else value
        assert np.array_equal(np.isnan(got), np.isnan(want)), np.argwhere(np.isnan(got) != np.isnan(want))[:5]
        assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]) and not np.isinf(got[~np.isinf(want)]).any()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [16, 5])
@pytest.mark.parametrize("h,new", [(4, 1), (4, 3), (24, 1), (24, 4)])
def test_attention_infinite_values_that_every_row_sees(kind, size, h, new):
    """They stay what they are, where weights are rounded too: alone, against a NaN,
    and with both signs."""
    g = gen(24)
    dtype, codes, d, kv, lens = kind.split()[0], "codes" in kind, 64, 2, [100, 700]
    table, pages = pages_of(g, lens, size)
    cache = Cache(g, pages, kv, size, d, dtype, codes)
    q = heads(g, len(lens) * new, h, d, dtype)
    inf, nan = float("inf"), float("nan")
    want = np.zeros((len(lens), kv, d))
    for b, j, head, c, value in [(0, 5, 0, 3, inf), (0, 40, 0, 9, -inf), (0, 41, 0, 9, -inf), (0, 63, 1, 20, inf),
                                 (0, 2, 1, 20, -inf), (1, 0, 0, 33, -inf), (1, 555, 1, 63, inf), (1, 31, 1, 0, inf),
                                 (1, 600, 1, 0, nan)]:
        pg, pl = place_of(table, size, b, j)
        if codes:      # (the format has no infinity; a scale of byte 255 makes a block of NaNs)
            cache.v[pg, head, pl, c // 32 * 32:c // 32 * 32 + 32] = 0x7F
            cache.vs[pg, head, pl, c // 32] = 255
            want[b, head, c // 32 * 32:c // 32 * 32 + 32] = nan
        else:
            cache.v[pg, head, pl, c] = value
            with np.errstate(invalid="ignore"):
                want[b, head, c] += value
    desc = fs.attention_desc(h, new, d ** -0.5)
    ws = torch.empty((fs.fs_paged_attention_workspace(desc, cache.struct, table) + 256,), dtype=torch.uint8, device=DEV)
    out = Out(len(lens) * new, h, d, dtype)
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    fs.fs_paged_attention(desc, cache.struct, q, lengths, table, out.view, ws)
    torch.cuda.synchronize()
    got = out.get().reshape(len(lens), new, kv, h // kv, d)
    want = np.broadcast_to(want[:, None, :, None], got.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    assert np.isfinite(got[np.isfinite(want)]).all()


def test_attention_scores_that_are_not_finite():
    """As the formula has them: a key of minus infinity has no weight, a row of
    nothing else is 0 / 0, a NaN or plus infinity makes NaNs."""
    g = gen(22)
    table, pages = pages_of(g, [20, 3], 16)
    for dtype in ("bf16", "f32"):
        cache = Cache(g, pages, 4, 16, 64, dtype)
        q = heads(g, 2, 4, 64, dtype)
        q[:, :, 0] = 1.0
        pg, pl = place_of(table, 16, 0, 7)
        cache.k[pg, 0, pl, 0] = float("-inf")
        cache.k[pg, 1, pl, 0] = float("inf")
        cache.k[pg, 2, pl, 5] = float("nan")
        for j in range(3):
            a, b = place_of(table, 16, 1, j)
            cache.k[a, 0, b, 0] = float("-inf")
        out, lse = torch.empty((2, 4, 64), dtype=TORCH[dtype], device=DEV), torch.empty((2, 4), device=DEV)
        lengths = torch.tensor([20, 3], dtype=torch.int32, device=DEV)
        fs.fs_paged_attention(fs.attention_desc(4, 1, 0.125), cache.struct, q, lengths, table, out, None, lse=lse)
        torch.cuda.synchronize()
        nan = torch.isnan(out).all(2).tolist()
        assert nan == [[False, True, True, False], [True, False, False, False]]
        assert torch.isfinite(out[0, 0]).all() and torch.isfinite(out[0, 3]).all()
        assert torch.isnan(lse[0, 1:3]).all() and lse[1, 0] == float("-inf") and torch.isfinite(lse[0, 0])


@pytest.mark.parametrize("lens", [[2500], [2500] + [40] * 70])
def test_attention_scores_that_are_not_finite_divided(lens):
    """The same where a sequence is in several parts: a NaN in one of them reaches
    its row, keys of minus infinity have no weight."""
    g = gen(23)
    table, pages = pages_of(g, lens, 16)
    cache = Cache(g, pages, 4, 16, 64, "bf16")
    q = heads(g, len(lens), 4, 64, "bf16")
    q[:, :, 0] = 1.0
    for j in range(1200):
        a, b = place_of(table, 16, 0, j)
        cache.k[a, 0, b, 0] = float("-inf")
    for h, j, value in ((1, 1300, "nan"), (2, 60, "inf")):
        a, b = place_of(table, 16, 0, j)
        cache.k[a, h, b, 0] = float(value)
    out, lse = torch.empty((len(lens), 4, 64), dtype=torch.bfloat16, device=DEV), torch.empty((len(lens), 4), device=DEV)
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    desc = fs.attention_desc(4, 1, 0.125)
    ws = torch.empty((fs.fs_paged_attention_workspace(desc, cache.struct, table),), dtype=torch.uint8, device=DEV)
    fs.fs_paged_attention(desc, cache.struct, q, lengths, table, out, ws, lse=lse)
    torch.cuda.synchronize()
    assert torch.isnan(out[0]).all(1).tolist() == [False, True, True, False] and torch.isfinite(out[0, [0, 3]]).all()
    assert torch.isnan(lse[0]).tolist() == [False, True, True, False] and torch.isfinite(out[1:]).all()
    k, v = cache.values()
    want = O.attention(f64(q)[:1, :1], k[:, :1], v[:, :1], lens[:1], table.cpu().numpy()[:1], 1, 0.125)[0]
    near(f64(out)[:1, :1], want, 2.0 ** -6 * np.abs(v).max())


def test_attention_lowest_values():
    """Scores at the type's lowest value: finite, and even ones share their weight."""
    low = torch.finfo(torch.float32).min
    table = torch.tensor([[0]], dtype=torch.int32, device=DEV)
    k, v = torch.zeros((1, 1, 16, 64), device=DEV), torch.randn((1, 1, 16, 64), generator=gen(1), device=DEV)
    k[0, 0, :, 0] = low
    q = torch.zeros((1, 1, 64), device=DEV)
    q[..., 0] = 1.0
    out, lse = torch.empty((1, 1, 64), device=DEV), torch.empty((1, 1), device=DEV)
    lengths = torch.tensor([16], dtype=torch.int32, device=DEV)
    fs.fs_paged_attention(fs.attention_desc(1, 1, 0.5), fs.kv_cache(k, v), q, lengths, table, out, None, lse=lse)
    torch.cuda.synchronize()
    near(f64(out)[0, 0], f64(v)[0, 0].mean(0), 32 * 2.0 ** -24 * np.abs(f64(v)[0, 0]).mean(0))


# ------------------------------------------------ far places, streams, graphs
@pytest.mark.parametrize("kind", ["bf16", "bf16 codes"])
def test_places_past_32_bits(kind):
    """Pages whose elements lie behind 2^32, of a cache that is mostly not touched."""
    dtype, codes = kind.split()[0], "codes" in kind
    kv, size, d = 8, 64, 128
    pages = (1 << 32) // (kv * size * d) + 40
    dt = torch.uint8 if codes else TORCH[dtype]
    k, v = (torch.empty((pages, kv, size, d), dtype=dt, device=DEV) for _ in range(2))
    scales = [torch.empty((pages, kv, size, 4), dtype=torch.uint8, device=DEV) for _ in range(2)] if codes else []
    cache = fs.kv_cache(k, v, *scales, dtype=dtype)
    g = gen(31)
    n = 300
    far = pages - 1 - torch.arange(5, dtype=torch.int32, device=DEV)[None]
    rows = [heads(g, n, kv, d, dtype) for _ in range(2)]
    pos, seqs = torch.arange(n, dtype=torch.int32, device=DEV), torch.zeros((n,), dtype=torch.int32, device=DEV)
    fs.fs_cache_append(cache, None, None, *rows, seqs, pos, far, None)
    q, lengths = heads(g, 1, 16, d, dtype), torch.tensor([n], dtype=torch.int32, device=DEV)
    out = torch.empty((1, 16, d), dtype=TORCH[dtype], device=DEV)
    desc = fs.attention_desc(16, 1, 0.1)
    ws = torch.empty((max(256, fs.fs_paged_attention_workspace(desc, cache, far)),), dtype=torch.uint8, device=DEV)
    fs.fs_paged_attention(desc, cache, q, lengths, far, out, ws)
    # the same in a cache of five pages
    near5 = torch.arange(4, -1, -1, dtype=torch.int32, device=DEV)[None]
    small = Cache(g, 5, kv, size, d, dtype, codes)
    fs.fs_cache_append(small.struct, None, None, *rows, seqs, pos, near5, None)
    out2 = torch.empty_like(out)
    fs.fs_paged_attention(desc, small.struct, q, lengths, near5, out2, ws)
    torch.cuda.synchronize()
    assert torch.equal(k[-5:][:, :, :n % 64], small.k[:, :, :n % 64])
    assert torch.equal(out, out2) and bool(torch.isfinite(out).all())


def serving(g, sequences=6, pages=40, dtype="bf16", codes=False, new=1, rope_layout="halves", d=96, hd=32, h=6, kv=2,
            size=8, window=0):
    """An attention sublayer, its cache and page table."""
    def w(m, n):
        return (torch.randn((m, n), generator=g, device=DEV) * n ** -0.5).to(TORCH[dtype])

    cache = fs.empty_cache(pages, size, kv, hd, dtype, codes)
    for t in cache.tensors:
        if t is not None:
            t.fill_(0x7F if t.dtype == torch.uint8 else float("nan"))
    freqs = fs.fs_rope_frequencies(hd).to(DEV)
    params = [1 + 0.1 * torch.randn((d,), generator=g, device=DEV), None, w((h + 2 * kv) * hd, d),
              0.1 * torch.randn(((h + 2 * kv) * hd,), generator=g, device=DEV), w(d, h * hd), None]
    table = torch.randperm(pages, generator=g, device=DEV).int()[:sequences * (pages // sequences)].view(sequences, -1)
    sub = fs.AttentionSublayer(sequences, cache, table.shape[1], *params, rope=fs.rope(freqs, rope_layout),
                               new_tokens=new, window=window)
    return sub, params, table, freqs


@pytest.mark.parametrize("window", [0, 5])
@pytest.mark.parametrize("kind", ["f32", "bf16", "bf16 codes"])
def test_sublayer(kind, window):
    """Tokens one after another, and several at once, through the sublayer: each
    pass's parts from what the part before it left, and the cache they left."""
    dtype, codes = kind.split()[0], "codes" in kind
    g = gen(41)
    B, d, hd, h, kv, size = 6, 96, 32, 6, 2, 8
    for new in (1, 4):
        sub, params, table, freqs = serving(g, B, 40, dtype, codes, new, window=window)
        tb = table.cpu().numpy()
        lens = np.array([0, 3, 0, 7, 1, 20])
        keys = {}
        for step in range(5):
            lens = lens + new
            lens[2] = 0                          # a sequence that is idle
            pos = (lens[:, None] - new + np.arange(new)).reshape(-1)
            pos[pos < 0] = -1
            x = torch.randn((B * new, d), generator=g, device=DEV).to(TORCH[dtype])
            out = torch.empty_like(x)
            lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
            if step == 0:                        # what came before this test's tokens
                for b in range(B):
                    n = int(lens[b]) - new
                    if n > 0:
                        rows = [heads(g, n, kv, hd, dtype) for _ in range(2)]
                        fs.fs_cache_append(sub.cache, None, None, *rows, torch.full((n,), b, dtype=torch.int32, device=DEV),
                                           torch.arange(n, dtype=torch.int32, device=DEV), table, None)
            sub.forward(x, out, torch.tensor(pos, dtype=torch.int32, device=DEV), lengths, table)
            torch.cuda.synchronize()
            qkv, q, o = (f64(t) for t in sub.heads)
            # the rotation
            live = pos >= 0
            want = O.rotary(qkv[:, :h], pos, freqs.cpu().numpy())
            tol = turn_tol(qkv[:, :h], freqs, "halves", 0, 1.0, want, dtype)
            near(q[live], want[live], tol[live])
            assert (q[~live] == 0).all()
            # the cache's new rows
            k, v, *sc = sub.cache.tensors
            kk, vv = ((f64(k), f64(v)) if not codes else
                      tuple(O.decoded(a.cpu().numpy(), b.cpu().numpy()) for a, b in zip((k, v), sc)))
            tk = O.rotary(qkv[:, h:h + kv], pos, freqs.cpu().numpy())
            tv = qkv[:, h + kv:]
            for t in np.flatnonzero(live):
                pg, pl = O.place(tb, 40, size, t // new, pos[t])
                if codes:
                    assert np.array_equal(vv[pg, :, pl], O.decoded(*O.coded(tv[t])))
                    assert np.abs(kk[pg, :, pl] - tk[t]).max() <= 2.0 ** -4 * np.abs(tk[t]).max() * (1 + 1e-6)
                else:
                    assert np.array_equal(vv[pg, :, pl], tv[t])
                    near(kk[pg, :, pl], tk[t], turn_tol(qkv[t, h:h + kv], freqs, "halves", 0, 1.0, tk[t], dtype))
                keys[(t // new, int(pos[t]))] = kk[pg, :, pl].copy()
            for (b, p), row in keys.items():     # those of earlier passes are still there
                pg, pl = O.place(tb, 40, size, b, p)
                assert np.array_equal(kk[pg, :, pl], row)
            # the attention, and the linear with the residual
            want, _, mass, reach = O.attention(q, kk, vv, lens, tb, new, float(np.float32(hd ** -0.5)), window)
            err = np.expm1((hd + 2) * U * reach) + 2.0 ** -21 + 40 * 2.0 ** -24 + 2.0 ** -20
            tol = (2 * (err + (2.0 ** -8 if dtype == "bf16" else 0)))[..., None] * mass
            near(o, want, tol + HALF[dtype] * (np.abs(want) + tol))
            W, flat = f64(params[4]), o.reshape(B * new, -1)
            want = f64(x) + flat @ W.T
            tol = (h * hd + 2) * U * (np.abs(flat) @ np.abs(W).T + np.abs(f64(x)))
            near(f64(out), want, tol + HALF[dtype] * (np.abs(want) + tol))


def test_sublayer_one_by_one_and_at_once():
    """Four tokens in one pass and one after another: in fp32 the same values to the
    roundings of sums in another order (a row of 96 or 192 terms, four times)."""
    g = gen(43)
    one, _, table, _ = serving(g, 6, 40, "f32")
    g = gen(43)
    four, _, table4, _ = serving(g, 6, 40, "f32", new=4)
    assert torch.equal(table, table4)
    x = torch.randn((6, 4, 96), generator=gen(44), device=DEV)
    out, outs = torch.empty((24, 96), device=DEV), []
    pos = torch.arange(4, dtype=torch.int32, device=DEV).repeat(6)
    four.forward(x.view(24, 96), out, pos, torch.full((6,), 4, dtype=torch.int32, device=DEV), table)
    for i in range(4):
        y = torch.empty((6, 96), device=DEV)
        one.forward(x[:, i].contiguous(), y, torch.full((6,), i, dtype=torch.int32, device=DEV),
                    torch.full((6,), i + 1, dtype=torch.int32, device=DEV), table)
        outs.append(y)
    torch.cuda.synchronize()
    want = torch.stack(outs, 1).view(24, 96)
    assert (out - want).norm() <= 4 * 192 * 2.0 ** -24 * want.norm()


def test_graph():
    """A captured step replayed, with eager work and synchronizations between,
    while lengths, positions and inputs change where they are."""
    g = gen(51)
    for new, codes in ((1, False), (3, True)):
        sub, _, table, _ = serving(g, 6, 60, "bf16", codes, new)
        for t in sub.cache.tensors:          # (tokens that no step here writes)
            if t is not None:
                t.fill_(0x38) if codes else t.normal_(generator=g)
        x, out = torch.empty((6 * new, 96), dtype=torch.bfloat16, device=DEV), torch.empty((6 * new, 96), dtype=torch.bfloat16, device=DEV)
        pos, lengths = torch.zeros((6 * new,), dtype=torch.int32, device=DEV), torch.zeros((6,), dtype=torch.int32, device=DEV)

        def step(n):
            x.normal_(generator=g)
            lengths.fill_(n)
            pos.copy_((n - new + torch.arange(new, device=DEV, dtype=torch.int32)).repeat(6))

        step(new)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            sub.forward(x, out, pos, lengths, table)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sub.forward(x, out, pos, lengths, table)
        for n in (new, 2 * new, 9 + new, 70, 71):
            step(n)
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            out.zero_()
            kept = [t.clone() for t in sub.cache.tensors if t is not None]
            sub.forward(x, out, pos, lengths, table)
            torch.cuda.synchronize()
            assert torch.equal(got, out)
            assert all(torch.equal(a, b) for a, b in zip(kept, [t for t in sub.cache.tensors if t is not None]))


def test_two_streams():
    """Calls at the same time on two streams, a workspace each."""
    g = gen(61)
    sets = []
    for seed in (1, 2):
        table, pages = pages_of(g, [900, 33, 2000], 16)
        cache = Cache(g, pages, 2, 16, 128, "bf16", codes=seed == 2)
        q = heads(g, 3, 8, 128, "bf16")
        desc = fs.attention_desc(8, 1, 0.1)
        ws = torch.empty((fs.fs_paged_attention_workspace(desc, cache.struct, table),), dtype=torch.uint8, device=DEV)
        sets.append((desc, cache, q, torch.tensor([900, 33, 2000], dtype=torch.int32, device=DEV), table, ws))
    want, got = [], []
    for desc, cache, q, lengths, table, ws in sets:
        out = torch.empty((3, 8, 128), dtype=torch.bfloat16, device=DEV)
        fs.fs_paged_attention(desc, cache.struct, q, lengths, table, out, ws)
        want.append(out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for s, (desc, cache, q, lengths, table, ws) in zip(streams, sets):
        outs = [torch.zeros((3, 8, 128), dtype=torch.bfloat16, device=DEV) for _ in range(8)]
        s.wait_stream(torch.cuda.current_stream())
        for out in outs:
            fs.fs_paged_attention(desc, cache.struct, q, lengths, table, out, ws, stream=s)
        got.append(outs)
    torch.cuda.synchronize()
    for w, outs in zip(want, got):
        assert all(torch.equal(w, o) for o in outs)


def test_graph_divided():
    """A captured call whose lengths change between replays, from nothing to what
    every workgroup has a part of, with eager calls on the same workspace between."""
    g = gen(71)
    lens = [2000, 1500, 0, 900, 2048]
    table, pages = pages_of(g, [2048] * 5, 16)
    for kind in ("bf16", "f32", "bf16 codes"):
        dtype, codes = kind.split()[0], "codes" in kind
        cache = Cache(g, pages, 2, 16, 128, dtype, codes)
        q = heads(g, 5, 6, 128, dtype)
        desc = fs.attention_desc(6, 1, 0.1)
        need = fs.fs_paged_attention_workspace(desc, cache.struct, table)
        assert need > 0
        ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)
        lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
        out, eager = (torch.empty((5, 6, 128), dtype=TORCH[dtype], device=DEV) for _ in range(2))
        lse = torch.empty((5, 6), device=DEV)
        fs.fs_paged_attention(desc, cache.struct, q, lengths, table, out, ws, lse=lse)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fs.fs_paged_attention(desc, cache.struct, q, lengths, table, out, ws, lse=lse)
        for step in ([0] * 5, [1, 0, 2048, 17, 16], lens, [2048] * 5, [3, 3, 3, 3, 3], lens):
            lengths.copy_(torch.tensor(step, dtype=torch.int32))
            out.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            fs.fs_paged_attention(desc, cache.struct, q, lengths, table, eager, ws)
            torch.cuda.synchronize()
            assert torch.equal(out, eager), step
            assert [bool(torch.isinf(r).all()) for r in lse] == [n == 0 for n in step]


# --------------------------------------------------- calls at the edges
def plain_call(cache, q, lengths, table, heads_, new=1, window=0):
    desc = fs.attention_desc(heads_, new, 0.125, window)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    lse = torch.full(q.shape[:2], 7.0, device=DEV)
    ws = torch.empty((max(256, fs.fs_paged_attention_workspace(desc, cache, table)),), dtype=torch.uint8, device=DEV)
    fs.fs_paged_attention(desc, cache, q, torch.tensor(lengths, dtype=torch.int32, device=DEV), table, out, ws, lse=lse)
    torch.cuda.synchronize()
    return out, lse


def test_lengths_out_of_range():
    """Negative lengths are 0, ones above the page table's reach end there."""
    g = gen(81)
    table, pages = pages_of(g, [600, 600, 600], 16)
    cache = Cache(g, pages, 2, 16, 64, "bf16")
    q = heads(g, 3, 4, 64, "bf16")
    reach = table.shape[1] * 16
    a = plain_call(cache.struct, q, [-5, 2 ** 31 - 1, -2 ** 31], table, 4)
    b = plain_call(cache.struct, q, [0, reach, 0], table, 4)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert bool((a[0][0] == 0).all()) and bool(torch.isfinite(a[1][1]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_there(dtype):
    """A page table without columns, a cache without pages, a step without rows."""
    g = gen(82)
    q = heads(g, 3, 4, 64, dtype)
    cache = Cache(g, 4, 2, 16, 64, dtype)
    none = torch.empty((3, 0), dtype=torch.int32, device=DEV)
    empty = fs.kv_cache(*(torch.empty((0, 2, 16, 64), dtype=TORCH[dtype], device=DEV) for _ in range(2)))
    table = torch.zeros((3, 40), dtype=torch.int32, device=DEV)
    for c, t in ((cache.struct, none), (empty, table), (empty, table[:, :3])):
        out, lse = plain_call(c, q, [5, 0, 600], t, 4)
        assert bool((out == 0).all()) and bool((lse == float("-inf")).all())
        before = cache.k.clone()
        k, v = heads(g, 3, 2, 64, dtype), heads(g, 3, 2, 64, dtype)
        pos = torch.tensor([0, 1, 700], dtype=torch.int32, device=DEV)
        qo = torch.empty_like(q)
        fs.fs_cache_append(c, None, q, k, v, None, pos, t, qo)
        torch.cuda.synchronize()
        assert torch.equal(qo, q) and torch.equal(cache.k, before)
    fs.fs_cache_append(cache.struct, None, None, k[:0], v[:0], None, pos[:0], table, None)
    fs.fs_rotary(fs.rotary_desc(0, 4, 64, dtype), None, q[:0], pos[:0], q[:0])
    out = torch.empty_like(q)
    fs.fs_rotary(fs.rotary_desc(3, 4, 64, dtype), None, q, pos, out)
    torch.cuda.synchronize()
    assert torch.equal(out, q)


def test_undivided_many_sequences():
    """More sequences than a divided call takes, one of them long."""
    g = torch.Generator().manual_seed(5)
    lens = torch.randint(0, 9, (4200,), generator=g).tolist()
    lens[4100] = 650
    check_attention("bf16", 1, 1, 64, lens, 16)


@pytest.mark.parametrize("size", [1, 5, 16])
@pytest.mark.parametrize("kind", ["bf16 codes", "f32 codes"])
@pytest.mark.parametrize("d", [8, 32, 72, 96, 136, 192, 200])
def test_last_scale_bytes(kind, d, size):
    """Every place of a cache in use: rows of few scale bytes at the end of theirs,
    which lie at the end of an allocation's part."""
    dtype = kind.split()[0]
    g = gen(83 + d)
    n = 80
    table, pages = pages_of(g, [n], size, spare=0)
    table.copy_(torch.arange(pages, dtype=torch.int32, device=DEV).flip(0) if size == 5 else torch.arange(pages, dtype=torch.int32, device=DEV))
    c = Cache(g, pages, 1, size, d, dtype, True)
    # the scales between bytes that would be seen as NaNs
    for x in (0, 1):
        s = (c.ks, c.vs)[x]
        full = torch.full((s.numel() + 512,), 255, dtype=torch.uint8, device=DEV)
        view = full[256:256 + s.numel()].view(s.shape)
        view.copy_(s)
        if x == 0:
            c.ks = view
        else:
            c.vs = view
    c.struct = fs.kv_cache(c.k, c.v, c.ks, c.vs, dtype=dtype)
    q = heads(g, 1, 2, d, dtype)
    out, lse = plain_call(c.struct, q, [n], table, 2)
    k, v = c.values()
    want, want_lse, mass, reach = O.attention(f64(q), k, v, [n], table.cpu().numpy(), 1, 0.125)
    err = np.expm1((d + 2) * U * reach) + 2.0 ** -21 + n * 2.0 ** -24 + 2.0 ** -20
    tol = (2 * (err + (2.0 ** -8 if dtype == "bf16" else 0)))[..., None] * mass
    near(f64(out), want, tol + HALF[dtype] * (np.abs(want) + tol))


def test_append_the_same_place_twice():
    """Every element is one of the two tokens', what is beside stays."""
    g = gen(84)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV)
    cache = Cache(g, 3, 2, 16, 64, "bf16")
    before = cache.k.clone()
    k, v = heads(g, 2, 2, 64, "bf16"), heads(g, 2, 2, 64, "bf16")
    at = torch.full((2,), 18, dtype=torch.int32, device=DEV)
    fs.fs_cache_append(cache.struct, None, None, k, v, torch.zeros_like(at), at, table, None)
    torch.cuda.synchronize()
    got = cache.k[0, :, 2]
    assert bool(((got == k[0]) | (got == k[1])).all())
    cache.k[0, :, 2] = before[0, :, 2]
    assert torch.equal(cache.k, before)


def test_keys_and_values_of_one_tensor():
    """A cache as [pages, 2, kv_heads, page, head_dim] and as [pages, page, 2,
    kv_heads, head_dim], against one of two tensors."""
    g = gen(85)
    table, pages = pages_of(g, [50, 33], 16)
    two = Cache(g, pages, 2, 16, 64, "bf16")
    q = heads(g, 2, 4, 64, "bf16")
    want = plain_call(two.struct, q, [50, 33], table, 4)
    one = torch.stack((two.k, two.v), 1)
    other = torch.stack((two.k.transpose(1, 2), two.v.transpose(1, 2)), 2).contiguous()
    for k, v in ((one[:, 0], one[:, 1]), (other[:, :, 0].transpose(1, 2), other[:, :, 1].transpose(1, 2))):
        got = plain_call(fs.kv_cache(k, v), q, [50, 33], table, 4)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ------------------------------------------------- weights of 16 bits more
@pytest.mark.parametrize("kind", ["bf16", "bf16 codes"])
@pytest.mark.parametrize("h,kv,d,new,lens,tokens", [
    (4, 2, 64, 1, [2, 4, 6, 10, 30, 600], 0), (8, 2, 128, 5, [6, 7, 10, 33], 0), (4, 2, 256, 1, [2, 4, 16, 40], 0),
    (36, 1, 64, 2, [3, 5, 9, 41], 70000), (36, 1, 128, 2, [3, 5, 9, 41], 70000), (24, 1, 256, 1, [2, 6, 20], 0),
    (128, 8, 64, 17, [17] * 8 + [24, 30], 0), (128, 8, 128, 17, [17] * 8 + [24, 30], 0)], ids=str)
def test_attention_weights_of_sixteen_bits(kind, h, kv, d, new, lens, tokens):
    """Pairs of tokens with almost the same key and opposite values: what is left of
    their sum shows the weights' roundings, 2^-16 of each (were they bf16 numbers,
    2^-9 of it would be left over).  One and several new tokens, four row tiles over
    a long table, prompts."""
    codes = "codes" in kind
    g = gen(91 + d)
    table, pages = pages_of(g, lens, 16, width=tokens // 16)
    cache = Cache(g, pages, kv, 16, d, "bf16", codes)
    cache.k[:, :, 1::2] = cache.k[:, :, ::2]
    # (the first column: 0, and 2^-5)
    cache.k[:, :, ::2, 0], cache.k[:, :, 1::2, 0] = (0, 0x10) if codes else (0.0, 2.0 ** -5)
    if codes:
        cache.v[:, :, 1::2] = cache.v[:, :, ::2] ^ 0x80
        cache.ks.fill_(127)
        cache.vs.fill_(127)
    else:
        cache.v[:, :, 1::2] = -cache.v[:, :, ::2]
    q = heads(g, len(lens) * new, h, d, "bf16")
    desc = fs.attention_desc(h, new, d ** -0.5)
    ws = torch.empty((fs.fs_paged_attention_workspace(desc, cache.struct, table) + 256,), dtype=torch.uint8, device=DEV)
    out = Out(len(lens) * new, h, d, "bf16")
    fs.fs_paged_attention(desc, cache.struct, q, torch.tensor(lens, dtype=torch.int32, device=DEV), table, out.view, ws)
    torch.cuda.synchronize()
    want, _, mass, reach = O.attention(f64(q), *cache.values(), lens, table.cpu().numpy(), new, float(np.float32(d ** -0.5)))
    err = np.expm1((d + 2) * U * reach) + 2.0 ** -21 + max(lens) * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -16
    tol = (2 * err)[..., None] * mass
    near(out.get(), want, tol + HALF["bf16"] * (np.abs(want) + tol))


# ----------------------------------------------- queries at places of their own
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("h,kv,d,new,window,size,lens", [
    (4, 2, 64, 1, 0, 16, [5, 700, 33, 0]), (4, 2, 128, 3, 0, 16, [5, 700, 33, 0]), (4, 2, 128, 3, 9, 7, [5, 700, 33, 0]),
    (12, 2, 72, 6, 40, 16, [90, 2, 300]), (20, 1, 64, 9, 0, 16, [900, 60]), (128, 8, 64, 17, 0, 16, [60, 17, 9] * 3 + [0]),
    (128, 8, 40, 17, 20, 5, [60, 17, 9] * 3 + [40])], ids=str)
def test_attention_at(kind, h, kv, d, new, window, size, lens):
    """Queries at any place, in any order, some of them none (their rows NaNs), some
    behind the last token; one token, several, row groups, a prompt's."""
    dtype, codes = kind.split()[0], "codes" in kind
    g = gen(95 + d + new)
    table, pages = pages_of(g, lens, size)
    cache = Cache(g, pages, kv, size, d, dtype, codes)
    t = len(lens) * new
    pos = torch.randint(-3, max(lens) + 5, (t,), generator=g, device=DEV, dtype=torch.int32).view(len(lens), new)
    pos[0, 0], pos[1, -1], pos[-1, 0] = -2 ** 31, 2 ** 31 - 1, -1
    if new > 1:
        pos[0, 0:] = torch.arange(new, device=DEV, dtype=torch.int32)      # from the start, the last none
        pos[0, -1:] = -1
    q = heads(g, t, h, d, dtype)
    last = np.repeat(lens, new) - 1
    at = np.minimum(pos.reshape(-1).cpu().numpy(), last)
    q[torch.tensor(at < 0, device=DEV)] = float("nan")
    desc = fs.attention_desc(h, new, d ** -0.5, window)
    ws = torch.empty((fs.fs_paged_attention_workspace(desc, cache.struct, table) + 256,), dtype=torch.uint8, device=DEV)
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out, lse = Out(t, h, d, dtype), torch.full((t, h), -77.0, device=DEV)
    fs.fs_paged_attention_at(desc, cache.struct, q, pos.reshape(-1), lengths, table, out.view, ws, lse=lse)
    torch.cuda.synchronize()
    tb = np.repeat(table.cpu().numpy(), new, axis=0)
    want, want_lse, mass, reach = O.attention(f64(q), *cache.values(), at + 1, tb, 1, float(np.float32(d ** -0.5)), window)
    err = np.expm1((d + 2) * U * reach) + 2.0 ** -21 + max(lens) * 2.0 ** -24 + 2.0 ** -20
    tol = (2 * (err + (2.0 ** -16 if dtype == "bf16" else 0)))[..., None] * mass
    near(out.get(), want, tol + HALF[dtype] * (np.abs(want) + tol))
    none = np.isneginf(want_lse)
    assert np.array_equal(none, np.isneginf(f64(lse))) and (out.get()[none] == 0).all()
    near(f64(lse)[~none], want_lse[~none], (2 * err + 2.0 ** -22 * np.abs(np.where(none, 0, want_lse)))[~none])
    # at the places that the sequences' last tokens have: the same bits as without
    q = torch.nan_to_num(q)
    ends = torch.clamp_min(lengths[:, None] - new + torch.arange(new, device=DEV, dtype=torch.int32), -1)
    a, b = Out(t, h, d, dtype), Out(t, h, d, dtype)
    fs.fs_paged_attention_at(desc, cache.struct, q, ends.int().reshape(-1), lengths, table, a.view, ws)
    fs.fs_paged_attention(desc, cache.struct, q, lengths, table, b.view, ws)
    torch.cuda.synchronize()
    assert np.array_equal(a.get(), b.get())


@pytest.mark.parametrize("window", [0, 5])
@pytest.mark.parametrize("side", ["last", "first", "between"])
def test_sublayer_padded_batch(side, window):
    """Ragged numbers of tokens, what is none of a sequence's rows last, first or in
    between: as one after another, in fp32 to the roundings of sums in another
    order (a row of 96 or 192 terms, four times)."""
    g = gen(46)
    one, _, table, _ = serving(g, 6, 40, "f32", window=window)
    g = gen(46)
    four, _, table4, _ = serving(g, 6, 40, "f32", new=4, window=window)
    assert torch.equal(table, table4)
    lens = torch.zeros((6,), dtype=torch.int32)
    for step, counts in enumerate([[4, 3, 2, 1, 0, 4], [1, 2, 4, 0, 3, 4], [4, 0, 1, 3, 2, 2]]):
        x = torch.randn((6, 4, 96), generator=gen(47 + step), device=DEV)
        pos = torch.full((6, 4), -1, dtype=torch.int32)
        for b, n in enumerate(counts):
            rows = {"last": range(n), "first": range(4 - n, 4), "between": [0, 2, 3, 1][:n]}[side]
            pos[b, sorted(rows)] = lens[b] + torch.arange(n, dtype=torch.int32)
        after = lens + torch.tensor(counts, dtype=torch.int32)
        out = torch.empty((24, 96), device=DEV)
        four.forward(x.view(24, 96), out, pos.view(-1).to(DEV), after.to(DEV), table)
        got = out.view(6, 4, 96)
        for i in range(4):
            live = (pos[:, i] >= 0).to(DEV)
            y = torch.empty((6, 96), device=DEV)
            now = torch.where(pos[:, i] >= 0, pos[:, i] + 1, lens).int()
            one.forward(x[:, i].contiguous(), y, pos[:, i].contiguous().to(DEV), now.to(DEV), table)
            torch.cuda.synchronize()
            assert (got[live, i] - y[live]).norm() <= 4 * 192 * 2.0 ** -24 * y[live].norm()
            assert torch.equal(got[~live, i], x[~live, i])          # (this sublayer has no b_out)
            lens = torch.where(pos[:, i] >= 0, pos[:, i] + 1, lens)
        assert torch.equal(lens.int(), after)


def test_attention_of_a_narrower_table():
    """The same call with a page table that is cut to the longest sequence, on the
    workspace of the whole one (of 33 rows a key head: with other row tiles): to the
    roundings of sums in another order."""
    g = gen(97)
    lens = [300, 7, 33, 0] * 10
    table, pages = pages_of(g, lens, 16, width=4375)
    cache = Cache(g, pages, 2, 16, 64, "bf16")
    q = heads(g, 40, 66, 64, "bf16")
    desc, lengths = fs.attention_desc(66, 1, 0.125), torch.tensor(lens, dtype=torch.int32, device=DEV)
    ws = torch.empty((fs.fs_paged_attention_workspace(desc, cache.struct, table),), dtype=torch.uint8, device=DEV)
    want, _, mass, reach = O.attention(f64(q), *cache.values(), lens, table.cpu().numpy()[:, :19], 1, 0.125)
    err = np.expm1(66 * U * reach) + 2.0 ** -21 + 300 * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -16
    tol = (2 * err)[..., None] * mass
    for width in (4375, 2047, 512, 33, 19):
        out = Out(40, 66, 64, "bf16")
        fs.fs_paged_attention(desc, cache.struct, q, lengths, table[:, :width], out.view, ws)
        torch.cuda.synchronize()
        near(out.get(), want, tol + HALF["bf16"] * (np.abs(want) + tol))


# ------------------------------------------------------- the ends of fp32's range
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 3])
def test_attention_scores_at_the_ends_of_the_range(dtype, new):
    """Scores of up to fp32's largest value: even ones share their weight, and of others
    the largest has it all; in a call of one part and in a divided one."""
    g = gen(98)
    big = float(torch.finfo(TORCH[dtype]).max)
    lens = [40, 33, 2000]
    table, pages = pages_of(g, lens, 16)
    for tokens in (40, 2000):
        cut = [min(n, tokens) for n in lens]
        for value, other in ((-big, None), (big, None), (big, -big), (0.9 * big, big), (-big, -0.9 * big)):
            cache = Cache(g, pages, 1, 16, 64, dtype)
            cache.k.fill_(0.0)
            cache.k[..., 0] = value
            top = [7, 30, 5]
            if other is not None:
                for b, j in enumerate(top):
                    pg, pl = place_of(table, 16, b, j)
                    cache.k[pg, 0, pl, 0] = other
            q = torch.zeros((3 * new, 2, 64), dtype=TORCH[dtype], device=DEV)
            q[..., 0] = 1.0
            desc = fs.attention_desc(2, new, 1.0)
            out = torch.empty((3 * new, 2, 64), dtype=TORCH[dtype], device=DEV)
            lse = torch.empty((3 * new, 2), device=DEV)
            pg = table[:, :(tokens + 15) // 16].contiguous()
            ws = torch.empty((fs.fs_paged_attention_workspace(desc, cache.struct, pg) + 256,), dtype=torch.uint8, device=DEV)
            fs.fs_paged_attention(desc, cache.struct, q, torch.tensor(cut, dtype=torch.int32, device=DEV), pg, out, ws, lse=lse)
            torch.cuda.synchronize()
            v = f64(cache.v)[:, 0]
            for b, n in enumerate(cut):
                for i in range(new):
                    at = n - new + i
                    rows = np.stack([v[place_of(table, 16, b, j)] for j in range(at + 1)])
                    if other is None:
                        seen, score = rows, value
                    elif other > value:
                        seen, score = rows[top[b]:top[b] + 1], other
                    else:
                        seen, score = np.delete(rows, top[b], 0), value
                    want = seen.mean(0)
                    tol = (2 * (len(seen) * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -16)) * np.abs(seen).mean(0)
                    near(f64(out)[b * new + i], np.broadcast_to(want, (2, 64)), tol + HALF[dtype] * (np.abs(want) + tol))
                    score = float(torch.tensor(score, dtype=TORCH[dtype]))
                    near(f64(lse)[b * new + i], np.full((2,), score), 2.0 ** -23 * abs(score))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("size", [16, 5])
@pytest.mark.parametrize("h,new", [(2, 1), (2, 3), (36, 1), (36, 2)])
def test_attention_infinite_values_of_small_weight(kind, size, h, new):
    """An infinite value stays one however far its score is below the largest (a weight
    that fp32 does not hold), in tiles that every row sees whole and in others, before
    and after the largest score, in the same part of a divided call and in another;
    finite ones there add nothing."""
    g = gen(99)
    inf, d = float("inf"), 64
    lens = [20, 100, 1500, 1500, 1500, 1500]
    table, pages = pages_of(g, lens, size, width=70000 // size)
    for below in (80.0, 95.0, 120.0, 1000.0, 2.0 ** 20):
        cache = Cache(g, pages, 1, size, d, kind)
        cache.k[..., 0] = 0.0
        cache.k[..., 1:] *= 0.01
        q = heads(g, len(lens) * new, h, d, kind)
        q[..., 0] = 1.0
        # (sequence, token of the infinite value, its column, token of the largest score)
        for b, j, c, top in [(0, 0, 3, 16), (1, 97, 9, 5), (2, 3, 20, 1400), (3, 1499 - new, 33, 2), (4, 700, 63, 703), (5, 60, 0, 30)]:
            pg, pl = place_of(table, size, b, top)
            cache.k[pg, 0, pl, 0] = below
            pg, pl = place_of(table, size, b, j)
            cache.v[pg, 0, pl, c] = inf if b % 2 else -inf
        out = Out(len(lens) * new, h, d, kind)
        # (short tables: few row tiles; long ones: many)
        for width in (1500 // size + 1, 70000 // size):
            t = table[:, :width]
            desc = fs.attention_desc(h, new, 1.0)
            ws = torch.empty((fs.fs_paged_attention_workspace(desc, cache.struct, t) + 256,), dtype=torch.uint8, device=DEV)
            fs.fs_paged_attention(desc, cache.struct, q, torch.tensor(lens, dtype=torch.int32, device=DEV), t, out.view, ws)
            torch.cuda.synchronize()
            got = out.get().reshape(len(lens), new, h, d)
            want = np.zeros((len(lens), d))
            for b, c in enumerate([3, 9, 20, 33, 63, 0]):
                want[b, c] = inf if b % 2 else -inf
            want = np.broadcast_to(want[:, None, None], got.shape)
            assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]), (below, width, got[np.isinf(want)][:8])
            assert np.isfinite(got[np.isfinite(want)]).all()
            k, v = cache.values()
            v = np.where(np.isfinite(v), v, 0.0)
            fine, _, mass, reach = O.attention(f64(q), k, v, lens, table.cpu().numpy()[:, :1501], new, 1.0)
            err = np.expm1((d + 2) * U * np.minimum(reach, 1000.0)) + 2.0 ** -20 + 1500 * 2.0 ** -24 + 2.0 ** -16
            tol = (2 * err)[..., None] * mass
            tol = (tol + HALF[kind] * (np.abs(fine) + tol)).reshape(got.shape)
            ok = np.isfinite(want)
            near(got[ok], fine.reshape(got.shape)[ok], tol[ok])


@pytest.mark.parametrize("new", [1, 4])
def test_sublayer_in_the_far_skip_window(new):
    """The sublayer as the next layer of a block: BEGIN, the sublayer on the partial
    input, FINISH into its output; twice, over the cache that grows.  The sublayer's
    part as by itself."""
    from workloads import CONFIGS, make_workload
    cfg = CONFIGS["tiny"]
    wl = make_workload(cfg, DEV)
    blk = fs.MoEBlock(cfg, wl.w_router, None, wl.w_gate_up, wl.w_down, device=DEV)
    n, d = cfg.n_tokens // new, cfg.hidden
    pair = [serving(gen(53), n, 3 * n, "f32", new=new, d=d)[:3:2] for _ in range(2)]
    (sub, table), (alone, table2) = pair
    assert torch.equal(table, table2)
    comm = torch.cuda.Stream()
    partial, out, by_itself, routed = (torch.empty_like(wl.x) for _ in range(4))
    for step in range(2):
        pos = (step * new + torch.arange(new, dtype=torch.int32, device=DEV)).repeat(n)
        lengths = torch.full((n,), (step + 1) * new, dtype=torch.int32, device=DEV)
        blk.begin(wl.x, partial, comm=comm)
        sub.forward(partial, out, pos, lengths, table)
        nxt = out.clone()
        blk.finish(wl.x, out, comm=comm)
        alone.forward(partial, by_itself, pos, lengths, table)
        L.fs_combine_unpack(blk.desc, blk.y_ret(), blk.t["slot_to_row"], blk.t["topk_w"], None, routed, None)
        torch.cuda.synchronize()
        assert torch.equal(nxt, by_itself) and torch.isfinite(out).all()
        # FINISH adds the routed output, one rounding
        both = f64(nxt) + f64(routed)
        near(f64(out), both, 4 * U * (np.abs(f64(nxt)) + np.abs(f64(routed))))
    blk.close()
