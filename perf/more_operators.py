"""Rotary positions and the paged 8-bit cache of a serving job as calls that can be timed and compared.

`own` false: the operators from elementary torch operations.  `own` true: the same through the
library's ctypes binding, as a program would call it.  A case's "op" names the operator, the other
entries are sizes and options; inputs are drawn on the GPU from the seed.

The cache: pages of `page` tokens of one sequence, K as [pages, kv_heads, page, dim] and V as
[pages, kv_heads, page / 16, dim, 16] bytes, each an e4m3 number; a byte e for each page and head says
that its numbers stand for 2^(e - 127) times as much.
"""
from __future__ import annotations

import math

import torch

own = False

BF16, F8, F64 = torch.bfloat16, torch.float8_e4m3fn, torch.float64


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # q and k of one token of a small model (768 hidden as 12 heads of 64): latency is everything
        dict(name="rope_token", op="rope", seqs=1, longest=1, heads=24, beside=12, dim=64, rot=64, layout="half", inverse=False, far=1024, factor=1.0),
        # a decode batch far into long contexts, a part of each head, neighbouring dims as pairs
        dict(name="rope_batch", op="rope", seqs=64, longest=1, heads=40, beside=8, dim=128, rot=64, layout="interleaved", inverse=False, far=1 << 20, factor=16.0),
        # a batch of prompts packed one behind the other, q and k of a fused projection with grouped heads
        dict(name="rope_prompts", op="rope", seqs=24, longest=4096, heads=40, beside=8, dim=128, rot=128, layout="half", inverse=False, far=32768, factor=4.0),
        # the gradient of a training step's queries (32 heads, sequences of 2048)
        dict(name="rope_back", op="rope", seqs=1, longest=4097, heads=32, beside=0, dim=128, rot=128, layout="half", inverse=True, far=8192, factor=1.0),
        # one token of one conversation
        dict(name="append_token", op="append", seqs=1, longest=1, held=1000, kv_heads=8, dim=128, page=64, rot=128, layout="half"),
        # a decode batch: a token for each of many conversations of all lengths, small pages
        dict(name="append_batch", op="append", seqs=64, longest=1, held=3001, kv_heads=8, dim=128, page=16, rot=64, layout="interleaved"),
        # prompts of every length, some of them behind what their conversation holds already
        dict(name="append_prompts", op="append", seqs=24, longest=4096, held=500, kv_heads=8, dim=128, page=64, rot=128, layout="half"),
        # one long document
        dict(name="append_long", op="append", seqs=1, longest=32768, held=0, kv_heads=8, dim=128, page=32, rot=128, layout="half"),
        # a few short conversations of a small model
        dict(name="paged_small", op="paged", batch=4, cap=512, heads=12, kv_heads=12, dim=64, page=16),
        # a serving batch of all lengths down to none
        dict(name="paged_batch", op="paged", batch=32, cap=4096, heads=32, kv_heads=8, dim=128, page=64),
        # seven query heads to a K/V head, lengths that end inside a page
        dict(name="paged_ragged", op="paged", batch=16, cap=3001, heads=28, kv_heads=4, dim=128, page=32),
        # long documents
        dict(name="paged_long", op="paged", batch=8, cap=131071, heads=32, kv_heads=8, dim=128, page=128),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step`, spread over the logarithm of [lo, hi]."""
    v = math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))
    return min(max(int(v / step + 0.5), (lo + step - 1) // step), max(hi, lo) // step) * step


def _draw_rope(rng):
    c = dict(op="rope", seqs=1 if rng.random() < 0.4 else _log(rng, 2, 256))
    c["heads"], c["beside"] = _log(rng, 1, 64), rng.choice([0, 0, 1, 8])
    c["dim"] = rng.choice([64, 80, 96, 128, 128, 256])
    c["rot"] = rng.choice([16, 32, c["dim"] // 2 // 16 * 16, c["dim"], c["dim"]])
    most = (1 << 24) // (c["heads"] * c["dim"])             # elements
    c["longest"] = max(1, _log(rng, 1, max(1, min(16384, most // (1 if c["seqs"] == 1 else c["seqs"] // 3 + 1)))))
    c["far"] = max(c["longest"], _log(rng, 1024, 1 << 21))
    return dict(c, layout=rng.choice(["half", "interleaved"]), inverse=rng.random() < 0.3, factor=rng.choice([1.0, 1.0, 4.0, 32.0]))


def _draw_append(rng):
    c = dict(op="append", seqs=1 if rng.random() < 0.3 else _log(rng, 2, 128), kv_heads=rng.choice([1, 2, 4, 5, 8, 12, 16, 32]),
             dim=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 128]))
    most = max(1, (1 << 18) // (c["kv_heads"] * c["seqs"]))  # tokens of a sequence
    c["longest"] = 1 if rng.random() < 0.3 else _log(rng, 1, min(16384, most))
    c["held"] = 0 if rng.random() < 0.3 else _log(rng, 1, min(8192, most))
    return dict(c, rot=rng.choice([0, 32, c["dim"] // 2, c["dim"], c["dim"]]), layout=rng.choice(["half", "interleaved"]))


def _draw_paged(rng):
    kv = rng.choice([1, 2, 4, 5, 8, 12, 16, 32])
    group = rng.choice([g for g in (1, 1, 2, 3, 4, 7, 8, 16, 32) if g * kv <= 64])
    c = dict(op="paged", batch=_log(rng, 1, 128), heads=kv * group, kv_heads=kv, dim=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 128]))
    return dict(c, cap=_log(rng, 1, max(1, min(131071, (1 << 22) // (c["batch"] * max(kv, group))))))


def draw(rng):
    return rng.choice([_draw_rope, _draw_append, _draw_paged])(rng)


# ---------------------------------------------------------------- sizes that follow from a case
def _lengths(c):
    """Tokens of the packed sequences: from 1 to the longest, spread over the logarithm."""
    n = c["seqs"]
    return [c["longest"]] if n == 1 else [int(c["longest"] ** (i / (n - 1)) + 0.5) for i in range(n)]


def _even(n, most):
    """From none to `most`, evenly (all of it, where there is one)."""
    return [most] if n == 1 else [most * i // (n - 1) for i in range(n)]


def _pages(tokens, page):
    return -(-tokens // page)


def work(c):
    if c["op"] == "rope":
        t = sum(_lengths(c))
        return dict(bytes=4 * t * c["heads"] * c["dim"] + 4 * t + 2 * c["rot"], flops=3 * t * c["heads"] * c["rot"])
    kv, d, page = c["kv_heads"], c["dim"], c["page"]
    if c["op"] == "append":
        t = sum(_lengths(c))
        pages = sum(_pages(n, page) for n in _lengths(c))
        return dict(bytes=6 * t * kv * d + pages * (4 + 2 * kv) + 8 * c["seqs"] + 2 * c["rot"], flops=t * kv * (3 * c["rot"] + 4 * d))
    t = sum(_even(c["batch"], c["cap"]))
    pages = sum(_pages(n, page) for n in _even(c["batch"], c["cap"]))
    return dict(bytes=2 * t * kv * d + pages * (4 + 2 * kv) + c["batch"] * (4 * c["heads"] * d + 4), flops=4 * t * c["heads"] * d)


# ---------------------------------------------------------------- what a program has in hand
class _Library:
    """One context with its two streams for the life of the process."""

    def __init__(self):
        self._ctx = None

    def context(self):
        import paper_2410_07381_amd.binding as B
        if self._ctx is None:
            self._ctx = B.Context(torch.cuda.Stream(), torch.cuda.Stream())
        return B, self._ctx


_LIB = _Library()


def _shuffled(values, gen):
    return torch.tensor(values, dtype=torch.int32)[torch.randperm(len(values), generator=gen)]


def _edges(lens):
    return torch.cat([torch.zeros(1, dtype=torch.int32), lens.cumsum(0).to(torch.int32)])


def _freqs(rot, factor=1.0):
    """Radians a position for each pair, positions pressed together by `factor`."""
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=F64) / max(rot, 1)) / factor).float().cuda()


def _table(tokens, page, spare, order):
    """Pages for sequences of so many tokens, in no order: [sequences, the longest's], and how many the pool has."""
    need = [_pages(n, page) for n in tokens]
    pool = sum(tokens) // page + len(tokens) + spare      # (enough however the tokens are spread)
    ids = torch.randperm(pool, generator=order).to(torch.int32)
    rows = torch.nn.utils.rnn.pad_sequence(list(ids[:sum(need)].split(need)), batch_first=True)
    return (rows if rows.shape[1] else rows.new_zeros((len(need), 1))).cuda(), pool


def _inputs(c, seed):
    """The inputs alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    order = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    def codes(*shape):                                    # numbers whose blocks reach towards 448
        return (normal(*shape) * 112).clamp_(-448, 448).to(F8).view(torch.uint8)

    def exps(pool, lo, hi):
        return torch.randint(lo, hi + 1, (pool, c["kv_heads"]), generator=g, device="cuda", dtype=torch.uint8)

    s = dict(case=c)
    if c["op"] == "rope":
        lens = _shuffled(_lengths(c), order)
        starts = (torch.rand(len(lens), generator=order, dtype=F64) * (c["far"] - lens + 1)).floor()
        s["positions"] = (torch.arange(int(lens.sum())) + (starts - _edges(lens)[:-1]).repeat_interleave(lens)).to(torch.int32).cuda()
        s["freqs"], s["magnitude"] = _freqs(c["rot"], c["factor"]), 1.0 + 0.1 * math.log(c["factor"])
        # (the heads to be rotated lie in front of others, as a fused projection leaves them)
        s["x"] = normal(int(lens.sum()), c["heads"] + c["beside"], c["dim"]).to(BF16)[:, :c["heads"]]
        return s
    kv, d, page = c["kv_heads"], c["dim"], c["page"]
    if c["op"] == "append":
        lens, held = _shuffled(_lengths(c), order), _shuffled(_even(c["seqs"], c["held"]), order)
        s["cu"], s["lens"] = _edges(lens).cuda(), (held + lens).cuda()   # (tokens with the new ones)
        s["kv"] = normal(int(lens.sum()), 2 * kv, d).to(BF16)
        s["freqs"] = _freqs(c["rot"]) if c["rot"] else None
        s["table"], pool = _table((held + lens).tolist(), page, 3, order)
        low, high = 119, 122
    else:
        lens = _shuffled(_even(c["batch"], c["cap"]), order)
        s["lens"] = lens.cuda()
        s["q"] = normal(c["batch"], c["heads"], d).to(BF16)
        s["table"], pool = _table(lens.tolist(), page, 3, order)
        low, high = 119, 120
    s["K"], s["V"] = codes(pool, kv, page, d), codes(pool, kv, page // 16, d, 16)
    s["Ke"], s["Ve"] = exps(pool, low, high), exps(pool, low, high)
    return s


def prepare(c, seed):
    s = _inputs(c, seed)
    if c["op"] == "rope":
        s["out"] = torch.zeros_like(s["x"], memory_format=torch.contiguous_format)
    elif c["op"] == "paged":
        s["out"] = torch.zeros_like(s["q"])
    if own:                                               # the descriptor of the call, which a program keeps
        B, _ = _LIB.context()
        if c["op"] == "rope":
            s["kernel"] = B.rope_bf16(s["x"], s["out"], s["freqs"], s["positions"], interleaved=c["layout"] == "interleaved",
                                      inverse=c["inverse"], magnitude=s["magnitude"])
            return s
        cache, kv = B.PagedCache(s["K"], s["V"], s["Ke"], s["Ve"]), c["kv_heads"]
        if c["op"] == "append":
            s["kernel"] = B.kv_append_fp8(s["kv"][:, :kv], s["kv"][:, kv:], s["cu"], s["lens"], s["table"], cache,
                                          freqs=s["freqs"], interleaved=c["layout"] == "interleaved")
        else:
            size = B.attn_paged_scratch_bytes(c["batch"], c["heads"], kv, c["dim"], c["page"], s["table"].shape[1])
            s["scratch"] = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
            s["kernel"] = B.attn_paged_fp8(s["q"], cache, s["table"], s["lens"], s["out"], s["scratch"])
    return s


# ---------------------------------------------------------------- the plain forms
def _rotated(x, positions, freqs, layout, sign=1.0):
    """x [tokens, heads, dim], its first 2 x freqs dims in pairs, by angles in 64 bits and in x's type otherwise."""
    n = freqs.numel()
    a = positions.double()[:, None, None] * freqs.double()
    c, s = a.cos().to(x.dtype), (sign * a.sin()).to(x.dtype)
    if layout == "half":
        p, q = x[..., :n], x[..., n:2 * n]
        return torch.cat([p * c - q * s, q * c + p * s, x[..., 2 * n:]], -1)
    p, q = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
    return torch.cat([torch.stack([p * c - q * s, q * c + p * s], -1).flatten(-2), x[..., 2 * n:]], -1)


def _plain_rope(s):
    c = s["case"]
    x = s["x"].float()
    n = c["rot"]
    out = _rotated(x, s["positions"], s["freqs"], c["layout"], -1.0 if c["inverse"] else 1.0)
    return torch.cat([out[..., :n] * s["magnitude"], out[..., n:]], -1).to(BF16)


def _two(e):
    """2^e in 64 bits, e a whole number."""
    return ((e.to(torch.int64) + 1023) << 52).view(F64)


def _e4m3(x):
    """The nearest e4m3 number, ties to even, of numbers in 64 bits up to 448 (rounded in 64 bits: by way of 32 a
    number next to a border would be rounded twice)."""
    step = _two(torch.frexp(x).exponent.clamp(min=-5) - 4)
    return (torch.round(x / step) * step).float().to(F8).view(torch.uint8)


def _blocks(x, row, off, new, codes, exps):
    """The codes and exponents of blocks [pages, heads, tokens, dims] in which the tokens `new` are x's: token i is in
    row[i], at place off[i]."""
    dense = torch.zeros(codes.shape, dtype=F64, device=x.device)
    dense[row.long(), :, off] = x
    part = torch.frexp(dense.abs().amax((2, 3)) / 448)
    need = torch.where(part.mantissa > 0.5, part.exponent, part.exponent - 1) + 127
    need = torch.where(part.mantissa == 0, torch.ones_like(need), need).clamp(1, 254)
    old = exps.to(torch.int32)
    e = torch.where(new[:, :1], need, torch.maximum(need, old))
    before = new.cumsum(1) == 0
    moved = _e4m3(codes.view(F8).double() * _two(old - e)[..., None, None])
    moved = torch.where(before[:, None, :, None], moved, codes)
    return torch.where(new[:, None, :, None], _e4m3(dense * _two(127 - e)[..., None, None]), moved), e.to(torch.uint8)


def _plain_append(s):
    c, cu, page, lens = s["case"], s["cu"], s["case"]["page"], s["lens"]
    kv, d = c["kv_heads"], c["dim"]
    at = torch.arange(s["kv"].shape[0], device=cu.device, dtype=torch.int32)
    seq = torch.searchsorted(cu[1:].contiguous(), at, right=True)
    place = lens[seq] - cu[seq + 1] + at
    # the pages that each sequence's new tokens lie in: rows enough for them from begin[i] on; the last page again where there are more
    first, begin = (lens - cu[1:] + cu[:-1]) // page, cu[:-1] // page + 2 * torch.arange(len(lens), device=cu.device, dtype=torch.int32)
    r = torch.arange(len(at) // page + 2 * len(lens), device=cu.device, dtype=torch.int32)
    of = torch.searchsorted(begin, r, right=True) - 1
    rows = begin[of] + torch.minimum(r - begin[of], (lens[of] - 1) // page - first[of])
    pages = s["table"][of, (first[of] + rows - begin[of]).long()].long()
    row, off = begin[seq] + place // page - first[seq], (place % page).long()
    new = torch.zeros((len(pages), page), dtype=torch.bool, device=cu.device)
    new[row.long(), off] = True
    k, v = s["kv"][:, :kv].double(), s["kv"][:, kv:].double()
    if c["rot"]:
        k = _rotated(k, place, s["freqs"], c["layout"])
    K, Ke = _blocks(k, row, off, new, s["K"][pages], s["Ke"][pages])
    V, Ve = _blocks(v, row, off, new, s["V"][pages].transpose(3, 4).reshape(-1, kv, page, d), s["Ve"][pages])
    s["K"][pages], s["Ke"][pages], s["Ve"][pages] = K[rows], Ke[rows], Ve[rows]
    s["V"][pages] = V[rows].view(-1, kv, page // 16, 16, d).transpose(3, 4)


def _values(codes, exps, table):
    """The numbers of the pages in a table's rows: [rows, pages of a row, heads, ...]."""
    at = table.long()
    return codes[at].view(F8).float() * _two(exps.to(torch.int32) - 127).float()[at].view(*at.shape, codes.shape[1], *[1] * (codes.dim() - 2))


def _plain_paged(s):
    c = s["case"]
    b, kv, d, group = c["batch"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"]
    keys = _values(s["K"], s["Ke"], s["table"]).permute(0, 2, 4, 1, 3).reshape(b, kv, d, -1)
    z = torch.matmul(s["q"].float().view(b, kv, group, d), keys).mul_(d ** -0.5)
    z.masked_fill_(torch.arange(z.shape[-1], device=z.device) >= s["lens"].view(b, 1, 1, 1), -math.inf)
    top = z.amax(-1, keepdim=True)
    p = z.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    values = _values(s["V"], s["Ve"], s["table"]).permute(0, 2, 1, 3, 5, 4).reshape(b, kv, -1, d)
    o = torch.matmul(p, values) / torch.where(total == 0, torch.ones_like(total), total)
    return o.reshape(b, c["heads"], d).to(BF16)


def run(s):
    c = s["case"]
    if own:
        _, ctx = _LIB.context()
        ctx.launch_native(s["kernel"], hi=True)
    elif c["op"] == "rope":
        return _plain_rope(s)
    elif c["op"] == "append":
        _plain_append(s)
    else:
        return _plain_paged(s)
    if c["op"] == "append":
        return [s["K"].view(F8), s["V"].view(F8), s["Ke"], s["Ve"]]
    return s["out"]


# ---------------------------------------------------------------- from the definition, in 64 bits
def _turned(x, positions, freqs, layout, sign=1):
    """Pairs as complex numbers."""
    n = freqs.numel()
    x = x.double()
    z = torch.complex(x[..., :n], x[..., n:2 * n]) if layout == "half" else torch.view_as_complex(x[..., :2 * n].unflatten(-1, (n, 2)).contiguous())
    angle = torch.outer(positions.double(), freqs.double())[:, None]
    z = z * torch.polar(torch.ones_like(angle), sign * angle)
    x = x.clone()
    if layout == "half":
        x[..., :n], x[..., n:2 * n] = z.real, z.imag
    else:
        x[..., 0:2 * n:2], x[..., 1:2 * n:2] = z.real, z.imag
    return x


def _numbers():
    """What each of the 256 codes stands for."""
    i = torch.arange(256, device="cuda")
    e, m = i // 8 % 16, (i % 8).double()
    x = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10).double())
    x[i % 128 == 127] = math.nan
    return torch.where(i < 128, x, -x)


def exact(c, seed):
    s = _inputs(c, seed)
    if c["op"] == "rope":
        x = _turned(s["x"], s["positions"], s["freqs"], c["layout"], -1 if c["inverse"] else 1)
        x[..., :c["rot"]] *= s["magnitude"]
        return x
    number, page, kv, d = _numbers(), c["page"], c["kv_heads"], c["dim"]
    table, lens = s["table"].tolist(), s["lens"].tolist()
    tokens_first = lambda v: v.permute(1, 3, 0, 2).reshape(page, kv, d)       # [heads, page / 16, dim, 16] of a page
    if c["op"] == "paged":
        out = torch.zeros(s["q"].shape, dtype=F64, device="cuda")
        for b, n in enumerate(lens):
            if n == 0:
                continue
            at = torch.tensor(table[b][:_pages(n, page)], device="cuda")
            for h in range(kv):
                k = (number[s["K"][at, h].long()] * 2.0 ** (s["Ke"][at, h].double() - 127).view(-1, 1, 1)).view(-1, d)[:n]
                v = number[s["V"][at, h].long()] * 2.0 ** (s["Ve"][at, h].double() - 127).view(-1, 1, 1, 1)
                v = v.transpose(2, 3).reshape(-1, d)[:n]
                g = slice(h * c["heads"] // kv, (h + 1) * c["heads"] // kv)
                e = s["q"][b, g].double() @ k.t() / math.sqrt(d)
                e = torch.exp(e - e.max(-1, keepdim=True).values)
                out[b, g] = e @ v / e.sum(-1, keepdim=True)
        return out
    # in units of each block's scale, and not rounded to 8 bits
    K, V, Ke, Ve = number[s["K"].long()], number[s["V"].long()], s["Ke"].long(), s["Ve"].long()
    limits = 448 * 2.0 ** (torch.arange(1, 254, dtype=F64, device="cuda") - 127)
    cu = s["cu"].tolist()
    for i, n in enumerate(lens):
        a, b = cu[i], cu[i + 1]
        k, v, first = s["kv"][a:b, :kv].double(), s["kv"][a:b, kv:].double(), n - (b - a)
        if c["rot"]:
            k = _turned(k, torch.arange(first, n, device="cuda"), s["freqs"], c["layout"])
        for p in range(first // page, _pages(n, page)):
            lo, hi = max(first, p * page), min(n, (p + 1) * page)
            at, cut, of = table[i][p], slice(lo - first, hi - first), lo - p * page
            values = tokens_first(V[at]).clone()
            for x, to, exps in ((k[cut], K[at].transpose(0, 1), Ke), (v[cut], values, Ve)):
                e = 1 + torch.searchsorted(limits, x.abs().amax((0, 2)))
                if of:
                    e = torch.maximum(e, exps[at])
                    to[:of] *= 2.0 ** (exps[at] - e).double()[:, None]
                to[of:of + hi - lo] = x * 2.0 ** (127 - e).double()[:, None]
                exps[at] = e
            V[at] = values.view(page // 16, 16, kv, d).permute(2, 0, 3, 1)
    return [K, V, Ke.to(torch.uint8), Ve.to(torch.uint8)]
