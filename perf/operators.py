"""The attention and 4-bit operators of a serving job as calls that can be timed and compared.

`own` false: the operators from elementary torch operations in 32 bits.  `own` true: the same
through the library's ctypes binding, as a program would call it.  A case's "op" names the
operator, the other entries are sizes and launch options; inputs are drawn on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

BF16 = torch.bfloat16


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # the prompt of one short request in a small model's layer (768 hidden as 12 heads of 64):
        # latency is everything
        dict(name="prompt_small", op="prompt", heads=12, kv_heads=12, dim=64, seqs=1, longest=128, behind=0, form="native"),
        # a batch of prompts of every length from one token up, packed one behind the other, with
        # grouped heads; some rows at the end of the buffers belong to nobody
        dict(name="prompt_packed", op="prompt", heads=32, kv_heads=8, dim=128, seqs=24, longest=4096, behind=37, form="native"),
        # the attention of a training-like step (32 heads, sequences of 2048) as a best-effort
        # client's persistent workers
        dict(name="prompt_workers", op="prompt", heads=32, kv_heads=32, dim=128, seqs=1, longest=4097, behind=0, form="ptb"),
        # one long document, all query heads on one K/V head
        dict(name="prompt_long", op="prompt", heads=8, kv_heads=1, dim=128, seqs=1, longest=32768, behind=0, form="native"),
        # four short conversations behind one system prompt, small model
        dict(name="prefix_small", op="prefix", batch=4, heads=12, kv_heads=12, dim=64, prefix=512, own_cap=64),
        # a serving batch behind a shared prompt, replies of every length down to none
        dict(name="prefix_batch", op="prefix", batch=32, heads=32, kv_heads=8, dim=128, prefix=4096, own_cap=512),
        # no shared part at all: a ragged batch of single-token queries, seven heads to a K/V head
        dict(name="prefix_none", op="prefix", batch=16, heads=28, kv_heads=4, dim=128, prefix=0, own_cap=3001),
        # a large batch that asks about one long document
        dict(name="prefix_long", op="prefix", batch=64, heads=32, kv_heads=8, dim=128, prefix=65500, own_cap=1024),
        # one token through a square projection: the smallest call there is
        dict(name="w4_token", op="w4", m=1, n=4096, k=4096, group=128, zeros=False),
        # one token through the larger of the feed-forward products
        dict(name="w4_ffn", op="w4", m=1, n=4096, k=11008, group=64, zeros=True),
        # a full batch of tokens through the other one
        dict(name="w4_batch", op="w4", m=16, n=11008, k=4096, group=128, zeros=False),
        # a vocabulary's logits for a ragged batch, small groups with zero points
        dict(name="w4_logits", op="w4", m=5, n=50257, k=4096, group=32, zeros=True),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step`, spread over the logarithm of [lo, hi]."""
    v = math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))
    return min(max(int(v / step + 0.5), (lo + step - 1) // step), max(hi, lo) // step) * step


def _draw_heads(rng):
    kv = rng.choice([1, 2, 4, 5, 8, 12, 16, 32])
    group = rng.choice([g for g in (1, 1, 2, 3, 4, 7, 8, 16) if g * kv <= 32])
    return dict(heads=kv * group, kv_heads=kv, dim=rng.choice([64, 128, 128]))


def _draw_prompt(rng):
    c = dict(op="prompt", **_draw_heads(rng))
    c["seqs"] = 1 if rng.random() < 0.4 else _log(rng, 2, 64)
    most = int(16384 * math.sqrt(32 / c["heads"]))        # scores of the plain form: heads x tokens^2
    if c["seqs"] > 1:
        most = min(most // 6, 8192)
    c["longest"] = _log(rng, 1 if c["seqs"] == 1 else 16, min(most, 32768))
    return dict(c, behind=rng.choice([0, 0, 1, 100]), form=rng.choice(["native", "native", "ptb"]))


def _draw_prefix(rng):
    c = dict(op="prefix", batch=_log(rng, 1, 128), **_draw_heads(rng))
    c["prefix"] = 0 if rng.random() < 0.15 else _log(rng, 1, min(65500, (1 << 27) // (c["batch"] * c["heads"])))
    rest = (1 << 19) // (c["batch"] * c["kv_heads"])
    c["own_cap"] = 0 if c["prefix"] and rng.random() < 0.15 else _log(rng, 1, max(1, min(8192, rest)))
    return c


def _draw_w4(rng):
    n = _log(rng, 48, 65536)
    return dict(op="w4", m=rng.choice([1, 1, 2, 3, 4, 8, 13, 16]), n=n, k=_log(rng, 64, min(16384, (1 << 27) // n), 8),
                group=rng.choice([32, 64, 128]), zeros=rng.random() < 0.5)


def draw(rng):
    return rng.choice([_draw_prompt, _draw_prefix, _draw_w4])(rng)


# ---------------------------------------------------------------- sizes that follow from a case
def _lengths(c):
    """Tokens of the packed sequences: from 1 to the longest, spread over the logarithm."""
    n = c["seqs"]
    return [c["longest"]] if n == 1 else [int(c["longest"] ** (i / (n - 1)) + 0.5) for i in range(n)]


def _replies(c):
    """Own tokens of the batch: evenly from none (one, where the batch has one row) to all of the cache."""
    n = c["batch"]
    return [c["own_cap"]] if n == 1 else [c["own_cap"] * i // (n - 1) for i in range(n)]


def work(c):
    if c["op"] == "prompt":
        t, pairs = sum(_lengths(c)), sum(n * (n + 1) // 2 for n in _lengths(c))
        return dict(bytes=2 * t * c["dim"] * (2 * c["heads"] + 2 * c["kv_heads"]) + 4 * (c["seqs"] + 1),
                    flops=4 * pairs * c["heads"] * c["dim"])
    if c["op"] == "prefix":
        t, pairs = c["prefix"] + sum(_replies(c)), c["batch"] * c["prefix"] + sum(_replies(c))
        return dict(bytes=4 * t * c["kv_heads"] * c["dim"] + 4 * c["batch"] * c["heads"] * c["dim"] + 4 * c["batch"],
                    flops=4 * pairs * c["heads"] * c["dim"])
    n, k = c["n"], c["k"]
    groups = -(-k // c["group"])
    return dict(bytes=n * k // 2 + n * groups * (3 if c["zeros"] else 2) + 2 * c["m"] * (n + k), flops=2 * c["m"] * n * k)


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


def _inputs(c, seed):
    """The inputs alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    order = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(BF16)

    s = dict(case=c)
    if c["op"] == "prompt":
        lens = _shuffled(_lengths(c), order)
        total = int(lens.sum()) + c["behind"]
        s["cu"] = torch.cat([torch.zeros(1, dtype=torch.int32), lens.cumsum(0).to(torch.int32)]).cuda()
        s["q"] = normal(total, c["heads"], c["dim"])
        # (one buffer for the two, as a fused projection leaves them)
        s["kv"] = normal(total, 2 * c["kv_heads"], c["dim"])
    elif c["op"] == "prefix":
        s["lens"] = _shuffled(_replies(c), order).cuda()
        s["q"] = normal(c["batch"], c["heads"], c["dim"])
        s["K"], s["V"] = (normal(c["prefix"], c["kv_heads"], c["dim"]) for _ in range(2))
        s["Ko"], s["Vo"] = (normal(c["batch"], c["own_cap"], c["kv_heads"], c["dim"]) for _ in range(2))
    else:
        n, k, m = c["n"], c["k"], c["m"]
        rows, blocks, groups = -(-n // 16), -(-k // 128), -(-k // c["group"])
        s["x"] = normal(m, k)
        # tiles of 16 rows by 128 weights: 64 lanes of four words of eight weights
        s["W"] = torch.randint(-(1 << 31), 1 << 31, (rows, blocks, 64, 4), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
        # (columns of 16 rows, one column per group)
        u = torch.rand((rows, groups, 16), generator=g, device="cuda")
        s["scales"] = ((0.5 + u) / (6.5 * math.sqrt(k))).to(BF16)
        s["zeros"] = torch.randint(4, 13, (rows, groups, 16), generator=g, device="cuda", dtype=torch.uint8) if c["zeros"] else None
    return s


def prepare(c, seed):
    s = _inputs(c, seed)
    if c["op"] == "w4":
        s["out"] = torch.zeros((c["m"], c["n"]), dtype=BF16, device="cuda")
    else:
        s["out"] = torch.zeros_like(s["q"])
    if own:                                               # the descriptor of the call, which a program keeps
        B, _ = _LIB.context()
        if c["op"] == "prompt":
            kv = c["kv_heads"]
            s["kernel"] = B.attn_prompt_bf16(s["q"], s["kv"][:, :kv], s["kv"][:, kv:], s["out"], s["cu"])
        elif c["op"] == "prefix":
            size = B.attn_prefix_scratch_bytes(c["batch"], c["heads"], c["kv_heads"], c["dim"], c["prefix"], c["own_cap"])
            s["scratch"] = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
            s["kernel"] = B.attn_prefix_bf16(s["q"], s["K"], s["V"], s["Ko"], s["Vo"], s["lens"], s["out"], s["scratch"])
        else:
            s["kernel"] = B.gemv_w4_bf16(s["x"], s["W"], s["scales"], s["out"], zeros=s["zeros"], group=c["group"])
    return s


# ---------------------------------------------------------------- the plain forms
def _attend(q, k, v, allowed, scale):
    """softmax(scale q k^T) v over the allowed pairs; rows that may attend to nothing give zeros."""
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(scale)
    s.masked_fill_(~allowed, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)


def _heads_first(t, repeat=1):
    t = t.float().transpose(0, 1)
    return t.repeat_interleave(repeat, 0).contiguous()


def _plain_prompt(s):
    c, q, cu = s["case"], s["q"], s["cu"]
    at = torch.arange(q.shape[0], device=q.device, dtype=torch.int32)
    seq = torch.searchsorted(cu[1:].contiguous(), at, right=True)
    inside = at < cu[-1]
    allowed = (seq[:, None] == seq[None, :]) & (at[None, :] <= at[:, None]) & inside[:, None]
    kv, group = c["kv_heads"], c["heads"] // c["kv_heads"]
    o = _attend(_heads_first(q), _heads_first(s["kv"][:, :kv], group), _heads_first(s["kv"][:, kv:], group), allowed,
                c["dim"] ** -0.5)
    return o.transpose(0, 1).to(BF16).contiguous()


def _plain_prefix(s):
    c = s["case"]
    b, kv, d, group = c["batch"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"]
    q = s["q"].float().view(b, kv, group, d)
    rows = q.transpose(0, 1).reshape(kv, b * group, d)
    shared = torch.matmul(rows, s["K"].float().permute(1, 2, 0).contiguous()).view(kv, b, group, c["prefix"]).transpose(0, 1)
    mine = torch.matmul(q, s["Ko"].float().permute(0, 2, 3, 1).contiguous())
    mine = mine.masked_fill(torch.arange(c["own_cap"], device=q.device) >= s["lens"].view(b, 1, 1, 1), -math.inf)
    z = torch.cat([shared, mine], -1) * d ** -0.5
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    near = p[..., c["prefix"]:]
    far = p[..., :c["prefix"]].transpose(0, 1).reshape(kv, b * group, c["prefix"])
    o = torch.matmul(far, s["V"].float().transpose(0, 1).contiguous()).view(kv, b, group, d).transpose(0, 1)
    o = o + torch.matmul(near, s["Vo"].float().transpose(1, 2).contiguous())
    return (o / torch.where(total == 0, torch.ones_like(total), total)).reshape(b, c["heads"], d).to(BF16)


def _weights(s, kind):
    """The weights as numbers, n x k.  Word i of lane 16 r + c of a tile holds row c's weights
    32 i + 8 r and the seven behind it, the even ones in its low half."""
    c = s["case"]
    shifts = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device="cuda", dtype=torch.int32)
    rows, blocks = s["W"].shape[:2]
    words = s["W"].view(rows, blocks, 4, 16, 4).permute(0, 3, 1, 4, 2)         # tile, row, block, i, r
    codes = (words[..., None] >> shifts) & 15
    codes = codes.reshape(rows * 16, blocks * 128)[:c["n"], :c["k"]]
    at = torch.arange(c["k"], device="cuda") // c["group"]
    scales = s["scales"].transpose(1, 2).reshape(rows * 16, -1)[:c["n"]].to(kind)[:, at]
    if s["zeros"] is None:
        return (codes - 8).to(kind) * scales
    zeros = s["zeros"].transpose(1, 2).reshape(rows * 16, -1)[:c["n"]].to(torch.int32)[:, at]
    return (codes - zeros).to(kind) * scales


def run(s):
    c = s["case"]
    if not own:
        if c["op"] == "prompt":
            return _plain_prompt(s)
        if c["op"] == "prefix":
            return _plain_prefix(s)
        return torch.matmul(s["x"].float(), _weights(s, torch.float32).t()).to(BF16)
    _, ctx = _LIB.context()
    if c.get("form") == "ptb":
        job = ctx.launch_ptb(s["kernel"], min(ctx.max_workers(s["kernel"]), s["kernel"].total_blocks))
        job.wait()
        job.free()
    else:
        ctx.launch_native(s["kernel"], hi=True)
    return s["out"]


# ---------------------------------------------------------------- from the definition, in 64 bits
def _softmax_sum(z, v):
    e = torch.exp(z - z.max(-1, keepdim=True).values)
    return (e @ v) / e.sum(-1, keepdim=True)


def exact(c, seed):
    s = _inputs(c, seed)
    if c["op"] == "w4":
        return torch.cat([s["x"].double() @ w.t() for w in _exact_weights(s)], 1)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group, root = c["heads"] // c["kv_heads"], math.sqrt(c["dim"])
    if c["op"] == "prompt":
        ends = s["cu"].tolist()
        for a, b in zip(ends, ends[1:]):
            hidden = torch.ones((b - a, b - a), dtype=torch.bool, device="cuda").triu(1)
            for h in range(c["heads"]):
                k, v = s["kv"][a:b, h // group].double(), s["kv"][a:b, c["kv_heads"] + h // group].double()
                z = s["q"][a:b, h].double() @ k.t() / root
                out[a:b, h] = _softmax_sum(z.masked_fill_(hidden, -math.inf), v)
        return out
    for i, n in enumerate(s["lens"].tolist()):
        if c["prefix"] + n == 0:
            continue
        k = torch.cat([s["K"], s["Ko"][i, :n]]).double().transpose(0, 1)       # kv_heads, tokens, dim
        v = torch.cat([s["V"], s["Vo"][i, :n]]).double().transpose(0, 1)
        q = s["q"][i].double().view(c["kv_heads"], group, c["dim"])
        out[i] = _softmax_sum(q @ k.transpose(1, 2) / root, v).reshape(c["heads"], c["dim"])
    return out


def _exact_weights(s):
    """Slabs of the weights in 64 bits, row tiles at a time, nibble by nibble."""
    c = s["case"]
    n, k = c["n"], c["k"]
    rows, blocks = s["W"].shape[:2]
    words = s["W"].to(torch.int64) & 0xFFFFFFFF
    for t in range(0, rows, 256):
        w = words[t:t + 256]
        tile = torch.zeros((w.shape[0], 16, blocks, 128), dtype=torch.float64, device="cuda")
        for r in range(4):
            for e in range(8):
                nib = (w[:, :, 16 * r:16 * r + 16] >> (4 * (e // 2) + 16 * (e % 2))) & 15   # tiles, blocks, 16, 4
                tile[:, :, :, 8 * r + e::32] = nib.permute(0, 2, 1, 3).double()
        tile = tile.reshape(-1, blocks * 128)[:, :k]
        of = [g // c["group"] for g in range(k)]
        zero = 8.0 if s["zeros"] is None else s["zeros"][t:t + 256].permute(0, 2, 1).reshape(tile.shape[0], -1)[:, of].double()
        tile = (tile - zero) * s["scales"][t:t + 256].permute(0, 2, 1).reshape(tile.shape[0], -1)[:, of].double()
        yield tile[:n - 16 * t]
