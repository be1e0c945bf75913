"""The attention sublayer's operators, as a program calls them: rotary positions
and their backward pass, appending keys and values to a paged cache with the
rotation on the way, and the attention of new tokens over that cache.

    listed()            the named cases
    draw(rng)           one more case of the same ranges
    prepare(case, s)    what a program holds before the call
    run(state)          one pass, and its outputs (``own``: by the library's
                        calls; else in plain torch operations)
    work(case)          bytes and flops the pass cannot do without
    exact(case, s)      the same outputs from the definitions, in 64 bits

A cache is [pages, kv_heads, page, head_dim].  Where it is held in 8 bits, an
append returns it as the values that it stands for (read back in the same pass).
"pad" adds so many elements to the stride between tokens.
"""

import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 32            # columns that share one scale of an 8-bit cache
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

ROTARY = dict(op="rotary", dtype="bf16", backward=False, layout="halves", first=0, scaling="plain", far=8192, pad=0)
APPEND = dict(op="append", dtype="bf16", codes=False, layout="halves", first=0, scaling="plain", page=16,
              skip=0, ragged=True, pad=0)
ATTEND = dict(op="attention", dtype="bf16", codes=False, new=1, page=16, window=0, ragged=True, empty=0, pad=0)


def listed():
    return [
        # a token of single-stream generation: the query and key heads of one
        # projection at the Llama-4-Scout-shaped hidden size
        dict(ROTARY, name="rotary_one_token", tokens=1, heads=48, d=128, rot=128),
        # a training step's queries and keys, frequencies scaled by parts for a
        # context longer than the trained one
        dict(ROTARY, name="rotary_train", tokens=8192, heads=48, d=128, rot=128, layout="pairs",
             scaling="parts", far=131072),
        # a training step's gradient where only the last 64 of a head's columns
        # carry the position
        dict(ROTARY, name="rotary_backward_part", tokens=4096, heads=128, d=192, rot=64, first=128, backward=True,
             layout="pairs"),
        # fp32 with sizes and strides that no vector divides (numerics checks)
        dict(ROTARY, name="rotary_odd", tokens=1001, heads=7, d=75, rot=38, first=3, dtype="f32", pad=5,
             scaling="linear"),
        # a serving step of 64 sequences, one new token each
        dict(APPEND, name="append_decode", seqs=64, new=1, start=512, heads=40, kv=8, d=128, rot=128),
        # two prompts into an 8-bit cache, read back
        dict(APPEND, name="append_prompt_8bit", seqs=2, new=4096, start=0, heads=40, kv=8, d=128, rot=128,
             codes=True, page=64, scaling="base"),
        # a padded batch with pages and heads of odd sizes, fp32
        dict(APPEND, name="append_odd", seqs=13, new=37, start=300, heads=6, kv=3, d=80, rot=40, first=16,
             dtype="f32", page=21, skip=3, pad=3, layout="pairs"),
        # single-stream generation at a short context
        dict(ATTEND, name="attention_one", seqs=1, length=1500, heads=40, kv=8, d=128, ragged=False),
        # a serving step of 64 sequences of very different lengths
        dict(ATTEND, name="attention_batch", seqs=64, length=8192, heads=40, kv=8, d=128),
        # a few long contexts in an 8-bit cache
        dict(ATTEND, name="attention_long_8bit", seqs=8, length=65536, heads=40, kv=8, d=128, page=64, codes=True),
        # four new tokens a sequence (a token and its drafts) with a sliding window
        dict(ATTEND, name="attention_drafts", seqs=32, length=16384, new=4, heads=64, kv=8, d=128, page=64,
             window=4096),
        # fp32, a key head for every query head, odd pages, idle sequences
        dict(ATTEND, name="attention_odd", seqs=9, length=2777, heads=11, kv=11, d=80, page=20, dtype="f32",
             empty=2, pad=7),
    ]


def draw(rng):
    def size(lo, hi, step=1):
        n = round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
        return min(hi, max(lo, n // step * step))

    op = rng.choice(("rotary", "rotary", "append", "append", "attention", "attention", "attention"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    pad = rng.choice((0, 0, 1, 8))
    scaling = rng.choice(("plain", "linear", "base", "parts"))
    layout = rng.choice(("halves", "pairs"))
    d = rng.choice((64, 80, 96, 128, 128, 128, 192, 256))
    if op == "rotary":
        if rng.random() < 0.3:
            d = rng.randint(16, 256)
        rot = rng.choice((d // 2 * 2, d // 4 * 2))
        heads, tokens = rng.randint(1, 64), size(1, 16384)
        while tokens * heads * d > 2 ** 26:
            tokens = tokens // 2
        return dict(ROTARY, dtype=dtype, tokens=tokens, heads=heads, d=d, rot=rot, layout=layout,
                    first=rng.choice((0, d - rot)), scaling=scaling, backward=rng.random() < 0.5,
                    far=size(100, 10 ** 6), pad=pad)
    kv = rng.choice((1, 2, 4, 8, 8, 11))
    heads = kv * rng.choice((1, 2, 4, 5, 8, 16))
    page = rng.choice((1, 7, 16, 16, 16, 20, 32, 64, 64, 256))
    codes = rng.random() < 0.4
    if op == "append":
        rot = rng.choice((d, d // 4 * 2))
        seqs, new = size(1, 256), size(1, 4096)
        while seqs * new * (heads + 2 * kv) * d > 2 ** 25:
            seqs, new = max(1, seqs // 2), max(1, new // 2)
        start = size(1, 1024)
        while seqs * (start + new) * kv * d > 2 ** 25 and start:
            start = start // 2
        return dict(APPEND, dtype=dtype, codes=codes, seqs=seqs, new=new, start=start,
                    heads=heads, kv=kv, d=d, rot=rot, first=rng.choice((0, d - rot)), layout=layout, page=page,
                    scaling=scaling, skip=rng.choice((0, 0, 1)), ragged=rng.random() < 0.7, pad=pad)
    seqs, length, new = size(1, 256), size(1, 131072), rng.choice((1, 1, 1, 2, 4, 7))
    while seqs * length * kv * d * max(1.0, heads * new / (8 * kv)) > 2 ** 27:
        seqs, length = max(1, seqs // 2), length // 2 + 1
    return dict(ATTEND, dtype=dtype, codes=codes, seqs=seqs, length=length, new=new, heads=heads, kv=kv, d=d,
                page=page, window=rng.choice((0, 0, 0, size(1, 8192))), ragged=rng.random() < 0.7,
                empty=rng.choice((0, 0, 1)), pad=pad)


# ------------------------------------------------------------------ inputs
def _lengths(n, most, ragged, empty=0):
    """Lengths of n sequences up to `most`, the first one the longest, spread
    over the range; every eighth is empty where `empty` says so."""
    out = []
    for i in range(n):
        x = 1.0 if i == 0 or not ragged else ((i * 0.6180339887) % 1.0) ** 1.5
        out.append(0 if empty and i % 8 == empty else max(1, round(most * x)))
    return out


def _frequencies(case):
    """[rot / 2] turning speeds in 64 bits, by the case's scaling for contexts
    eight times as long as trained (4096)."""
    r, base, factor, trained, lo, hi = case["rot"], 10000.0, 8.0, 4096.0, 1.0, 4.0
    i = torch.arange(r // 2, dtype=torch.float64)
    if case["scaling"] == "base" and r > 2:
        base *= factor ** (r / (r - 2))
    f = base ** (-2.0 * i / max(r, 1))
    if case["scaling"] == "linear":
        f = f / factor
    elif case["scaling"] == "parts":
        keep = ((trained * f / (2 * math.pi) - lo) / (hi - lo)).clamp(0, 1)
        f = f * (keep + (1 - keep) / factor)
    return f.to(DEV)


def _mscale(case):
    return 1.0 + 0.1 * math.log(8.0) if case["scaling"] == "parts" else 1.0


def _heads(gen, tokens, heads, case, scale=1.0):
    """[tokens, heads, d] of N(0, scale^2), as heads of a wider row."""
    d = case["d"]
    full = torch.empty((tokens, heads * d + case["pad"]), dtype=DTYPES[case["dtype"]], device=DEV)
    full.normal_(0.0, scale, generator=gen)
    return full[:, :heads * d].unflatten(1, (heads, d))


def _pages(gen, lens, case):
    """A page table: every sequence's pages, in any order over the cache."""
    p = case["page"]
    counts = [(n + p - 1) // p for n in lens]
    most, total = max(1, max(counts)), max(1, sum(counts))
    order = torch.randperm(total, generator=gen, device=DEV).int()
    table = torch.full((len(lens), most), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    return table, total


def _cache(gen, pages, case):
    """Keys and values of earlier tokens: a few channels of the keys are much
    larger than the rest."""
    shape = (pages, case["kv"], case["page"], case["d"])
    dt = torch.bfloat16 if case["codes"] else DTYPES[case["dtype"]]
    k = torch.empty(shape, dtype=dt, device=DEV).normal_(0.0, 1.0, generator=gen)
    v = torch.empty(shape, dtype=dt, device=DEV).normal_(0.0, 1.0, generator=gen)
    chan = torch.rand((case["d"],), generator=gen, device=DEV)
    k *= torch.where(chan < 0.03, 6.0, 0.7).to(dt)
    return k, v


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    c = case
    s = {"case": c, "keep": {}}
    if c["op"] == "rotary":
        s["x"] = _heads(gen, c["tokens"], c["heads"], c)
        s["positions"] = torch.randint(0, c["far"], (c["tokens"],), generator=gen, device=DEV, dtype=torch.int32)
        s["freqs"] = _frequencies(c)
        return s
    if c["op"] == "append":
        starts = [n - 1 for n in _lengths(c["seqs"], c["start"] + 1, c["ragged"])]
        t = c["seqs"] * c["new"]
        seqs = torch.arange(c["seqs"], device=DEV, dtype=torch.int32).repeat_interleave(c["new"])
        pos = torch.tensor(starts, device=DEV, dtype=torch.int32)[:, None] + torch.arange(
            c["new"], device=DEV, dtype=torch.int32)
        if c["skip"]:
            # a padded batch: the last tokens of every second sequence are none
            pos[1::2, max(1, c["new"] - c["skip"]):] = -1
        s["seqs"], s["positions"] = seqs, pos.reshape(-1).contiguous()
        s["live"] = (s["positions"] >= 0).nonzero()[:, 0]
        s["freqs"] = _frequencies(c)
        qkv = _heads(gen, t, c["heads"] + 2 * c["kv"], c)
        s["q"], s["k"], s["v"] = qkv.split((c["heads"], c["kv"], c["kv"]), dim=1)
        s["table"], pages = _pages(gen, [n + c["new"] for n in starts], c)
    else:
        s["lens"] = _lengths(c["seqs"], c["length"], c["ragged"], c["empty"])
        s["lengths"] = torch.tensor(s["lens"], device=DEV, dtype=torch.int32)
        s["q"] = _heads(gen, c["seqs"] * c["new"], c["heads"], c)
        s["table"], pages = _pages(gen, s["lens"], c)
    s["kc"], s["vc"] = _cache(gen, pages, c)
    if c["codes"]:
        s["kc"], s["vc"] = _encode(s["kc"]), _encode(s["vc"])
    return s


# -------------------------------------------------------------- plain form
def _pow2(e):
    """2^e in fp32, exactly, by its exponent field."""
    return ((e + 127).int() << 23).view(torch.float32)


def _encode(x):
    """Codes [..., d] and scale bytes [..., ceil(d / 32)] of an 8-bit cache."""
    d = x.shape[-1]
    nb = (d + BLOCK - 1) // BLOCK
    v = torch.nn.functional.pad(x.float(), (0, nb * BLOCK - d)).unflatten(-1, (nb, BLOCK))
    frac, exp = torch.frexp(v.abs().amax(-1))
    e = torch.clamp_min(exp - torch.where(frac <= 0.875, 9, 8), -117)
    codes = (v * _pow2(-e).unsqueeze(-1)).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes.flatten(-2)[..., :d].contiguous(), (e + 127).to(torch.uint8)


def _decode(codes, scales):
    """The fp32 values of an 8-bit cache (exact)."""
    v = codes.view(torch.float8_e4m3fn).float()
    return v * _pow2(scales.int() - 127).repeat_interleave(BLOCK, dim=-1)[..., :codes.shape[-1]]


def _values(t):
    return _decode(*t) if isinstance(t, tuple) else t.float()


def _turned(x, s, back=False):
    """x [tokens, heads, d] in fp32 with the case's columns turned."""
    c = s["case"]
    r, f = c["rot"], c["first"]
    angle = s["positions"].double()[:, None] * s["freqs"]
    cos = (torch.cos(angle) * _mscale(c)).float()[:, None]
    sin = (torch.sin(angle) * (-_mscale(c) if back else _mscale(c))).float()[:, None]
    out = x.float().clone()
    part = out[..., f:f + r]
    a, b = (part[..., :r // 2], part[..., r // 2:]) if c["layout"] == "halves" else (part[..., ::2], part[..., 1::2])
    na, nb = a * cos - b * sin, b * cos + a * sin
    a.copy_(na)
    b.copy_(nb)
    return out


def _plain(s):
    c = s["case"]
    dt = DTYPES[c["dtype"]]
    if c["op"] == "rotary":
        return {"out": _turned(s["x"], s, c["backward"]).to(dt)}
    if c["op"] == "append":
        live = s["live"]
        q = torch.zeros(s["q"].shape, dtype=dt, device=DEV)
        q[live] = _turned(s["q"], s).to(dt)[live]
        pos = s["positions"].long()[live]
        page, place = s["table"][s["seqs"].long()[live], pos // c["page"]].long(), pos % c["page"]
        out = {"q": q}
        for name, rows in (("k", _turned(s["k"], s)), ("v", s["v"].float())):
            cache = s[name + "c"]
            new = _encode(rows) if c["codes"] else (rows.to(dt),)
            for dst, src in zip(cache if c["codes"] else (cache,), new):
                dst[page, :, place] = src[live]
            out[name] = _decode(*cache).to(dt) if c["codes"] else cache
        return out
    n, g, kv, d = c["new"], c["heads"] // c["kv"], c["kv"], c["d"]
    o = torch.zeros((c["seqs"] * n, c["heads"], d), dtype=torch.float32, device=DEV)
    lse = torch.full((c["seqs"] * n, c["heads"]), -math.inf, dtype=torch.float32, device=DEV)
    for b, length in enumerate(s["lens"]):
        if length == 0:
            continue
        pages = s["table"][b, :(length + c["page"] - 1) // c["page"]].long()
        k, v = ((_decode(t[0][pages], t[1][pages]) if c["codes"] else t[pages].float())
                .transpose(0, 1).reshape(kv, -1, d)[:, :length] for t in (s["kc"], s["vc"]))
        q = s["q"][b * n:(b + 1) * n].float().unflatten(1, (kv, g)).permute(1, 0, 2, 3).reshape(kv, n * g, d)
        at = length - n + torch.arange(n, device=DEV)[:, None]
        j = torch.arange(length, device=DEV)
        seen = j <= at
        if c["window"]:
            seen &= j > at - c["window"]
        scores = (q @ k.transpose(1, 2)) * d ** -0.5
        scores = torch.where(seen.repeat_interleave(g, 0), scores, scores.new_full((), -math.inf))
        top = scores.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        p = torch.exp(scores - top)
        total = p.sum(-1, keepdim=True)
        rows = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
        o[b * n:(b + 1) * n] = rows.view(kv, n, g, d).permute(1, 0, 2, 3).reshape(n, -1, d)
        lse[b * n:(b + 1) * n] = (top + torch.log(total)).view(kv, n, g).permute(1, 0, 2).reshape(n, -1)
    return {"out": o.to(dt), "lse": lse}


# ------------------------------------------------------- the library's calls
def _kept(s, name, make):
    """What the program keeps from pass to pass: workspace, descriptor, outputs."""
    if name not in s["keep"]:
        s["keep"][name] = make()
    return s["keep"][name]


def _call(s):
    import paper_2511_11505_amd as fs

    c = s["case"]
    dt = DTYPES[c["dtype"]]

    def empty(name, shape, dtype=dt):
        return _kept(s, name, lambda: torch.empty(shape, dtype=dtype, device=DEV))

    def cache():
        if c["codes"]:
            return fs.kv_cache(s["kc"][0], s["vc"][0], s["kc"][1], s["vc"][1], dtype=c["dtype"])
        return fs.kv_cache(s["kc"], s["vc"], dtype=c["dtype"])

    def rope():
        return fs.rope(s["freqs"], layout=c["layout"], first=c["first"], mscale=_mscale(c))

    if c["op"] == "rotary":
        desc = _kept(s, "desc", lambda: fs.rotary_desc(c["tokens"], c["heads"], c["d"], c["dtype"]))
        out = empty("out", (c["tokens"], c["heads"], c["d"]))
        call = fs.fs_rotary_backward if c["backward"] else fs.fs_rotary
        call(desc, _kept(s, "rope", rope), s["x"], s["positions"], out)
        return {"out": out}
    if c["op"] == "append":
        q = empty("q", (c["seqs"] * c["new"], c["heads"], c["d"]))
        fs.fs_cache_append(_kept(s, "cache", cache), _kept(s, "rope", rope), s["q"], s["k"], s["v"], s["seqs"],
                           s["positions"], s["table"], q)
        out = {"q": q}
        for name in ("k", "v"):
            if c["codes"]:
                codes, scales = s[name + "c"]
                rows, d = codes.numel() // c["d"], c["d"]
                out[name] = empty(name, codes.shape)
                fs.fs_checkpoint_restore(fs.FS_BF16 if c["dtype"] == "bf16" else fs.FS_F32, rows, d,
                                         codes.view(rows, d), scales.view(rows, -1), out[name].view(rows, d))
            else:
                out[name] = s[name + "c"]
        return out
    desc = _kept(s, "desc", lambda: fs.attention_desc(c["heads"], c["new"], c["d"] ** -0.5, c["window"]))
    kv = _kept(s, "cache", cache)
    ws = _kept(s, "ws", lambda: torch.empty((max(256, fs.fs_paged_attention_workspace(desc, kv, s["table"])),),
                                            dtype=torch.uint8, device=DEV))
    out = empty("out", (c["seqs"] * c["new"], c["heads"], c["d"]))
    lse = empty("lse", (c["seqs"] * c["new"], c["heads"]), torch.float32)
    fs.fs_paged_attention(desc, kv, s["q"], s["lengths"], s["table"], out, ws, lse=lse)
    return {"out": out, "lse": lse}


def run(state):
    if own:
        return _call(state)
    return _plain(state)


# ----------------------------------------------------------- work and oracle
def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    d = c["d"]
    if c["op"] == "rotary":
        n = c["tokens"] * c["heads"] * d
        return {"bytes": 2 * e * n + 4 * c["tokens"] + 4 * c["rot"], "flops": 3.0 * c["tokens"] * c["heads"] * c["rot"]}
    row = d + (d + BLOCK - 1) // BLOCK if c["codes"] else e * d
    if c["op"] == "append":
        t, kv = c["seqs"] * c["new"], c["kv"]
        b = t * (2 * e * c["heads"] * d + 2 * kv * (e * d + row) + 12)
        if c["codes"]:
            # the cache is read back whole
            tokens = sum((n - 1 + c["new"] + c["page"] - 1) // c["page"] * c["page"]
                         for n in _lengths(c["seqs"], c["start"] + 1, c["ragged"]))
            b += 2 * tokens * kv * (row + e * d)
        return {"bytes": b, "flops": 3.0 * t * (c["heads"] + kv) * c["rot"]}
    rows = tokens = 0
    for n in _lengths(c["seqs"], c["length"], c["ragged"], c["empty"]):
        first = max(0, n - c["new"])
        tokens += n - (max(0, first + 1 - c["window"]) if c["window"] else 0)
        for at in range(n - c["new"], n):
            rows += max(0, min(at + 1, c["window"]) if c["window"] else at + 1)
    b = 2 * tokens * c["kv"] * row + c["seqs"] * c["new"] * c["heads"] * (2 * e * d + 4) + 8 * c["seqs"]
    return {"bytes": b, "flops": 4.0 * rows * c["heads"] * d}


def _f64_saved(t):
    """Values of a cache; each code decoded from its bits."""
    if not isinstance(t, tuple):
        return t.double()
    codes, scales = t
    field, man = (codes.int() >> 3) & 15, (codes & 7).double()
    mag = torch.where(field == 0, man / 8 * 2.0 ** -6, (1 + man / 8) * 2.0 ** (field.double() - 7))
    col = torch.arange(codes.shape[-1], device=codes.device) // BLOCK
    return torch.where(codes >= 128, -mag, mag) * 2.0 ** (scales[..., col].double() - 127)


def _f64_coded(x):
    """x [..., d] (64 bits) through 8 bits, by arithmetic on the code's grid."""
    d = x.shape[-1]
    v = torch.nn.functional.pad(x, (0, -d % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = v.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.clamp_min(top, 1e-300) / 448))
    e = torch.where(top > 448 * 2.0 ** e, e + 1, e)
    e = torch.where(top <= 448 * 2.0 ** (e - 1), e - 1, e).clamp_min(-117)
    q = v * 2.0 ** -e
    grid = 2.0 ** (torch.floor(torch.log2(torch.clamp_min(q.abs(), 2.0 ** -6))) - 3)
    return (torch.round(q / grid) * grid * 2.0 ** e).flatten(-2)[..., :d]


def _f64_turned(x, s, back=False):
    """The rotation as a product with each pair's complex number."""
    c = s["case"]
    r, f = c["rot"], c["first"]
    if c["layout"] == "halves":
        at = torch.stack((torch.arange(r // 2), torch.arange(r // 2) + r // 2), 1) + f
    else:
        at = torch.arange(r).view(-1, 2) + f
    at = at.to(x.device)
    angle = torch.outer(s["positions"].double(), s["freqs"]) * (-1 if back else 1)
    unit = torch.polar(torch.full_like(angle, _mscale(c)), angle)[:, None]
    out = x.double()
    z = torch.complex(out[..., at[:, 0]], out[..., at[:, 1]]) * unit
    out = out.index_copy(-1, at[:, 0], z.real)
    return out.index_copy(-1, at[:, 1], z.imag)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "rotary":
        return {"out": _f64_turned(s["x"], s, c["backward"])}
    if c["op"] == "append":
        q = _f64_turned(s["q"], s)
        q[s["positions"] < 0] = 0.0
        out = {"q": q}
        idx = torch.tensor([i for i, p in enumerate(s["positions"].tolist()) if p >= 0], device=DEV)
        place = s["positions"].long()[idx]
        seq = s["seqs"].long()[idx]
        page = s["table"].long()[seq, place // c["page"]]
        for name in ("k", "v"):
            cache = _f64_saved(s[name + "c"])
            rows = _f64_turned(s[name], s) if name == "k" else s[name].double()
            rows = _f64_coded(rows) if c["codes"] else rows
            flat = cache.transpose(1, 2).reshape(-1, c["kv"], c["d"])
            flat[page * c["page"] + place % c["page"]] = rows[idx]
            out[name] = flat.view(-1, c["page"], c["kv"], c["d"]).transpose(1, 2)
        return out
    n, h, kv, d = c["new"], c["heads"], c["kv"], c["d"]
    out = torch.zeros((c["seqs"], n, h, d), dtype=torch.float64, device=DEV)
    lse = torch.full((c["seqs"], n, h), -math.inf, dtype=torch.float64, device=DEV)
    q = s["q"].double().unflatten(0, (c["seqs"], n))
    for b in range(c["seqs"]):
        length = s["lens"][b]
        ids = torch.arange(length, device=DEV)
        page = s["table"].long()[b, ids // c["page"]]
        k, v = (_f64_saved(tuple(x[page, :, ids % c["page"]] for x in t) if c["codes"]
                           else t[page, :, ids % c["page"]]) for t in (s["kc"], s["vc"]))
        for i in range(n):
            hi = length - n + i + 1
            lo = max(0, hi - c["window"]) if c["window"] else 0
            if hi <= lo:
                continue
            for m in range(kv):
                heads = slice(m * (h // kv), (m + 1) * (h // kv))
                sc = q[b, i, heads] @ k[lo:hi, m].T / math.sqrt(d)
                lse[b, i, heads] = torch.logsumexp(sc, 1)
                out[b, i, heads] = torch.softmax(sc, 1) @ v[lo:hi, m]
    return {"out": out.flatten(0, 1), "lse": lse.flatten(0, 1)}
