"""What lies between a decoder block's fused QKV projection and its attention output projection.

Four kinds of work, as a program that serves such a block calls them:

  rotate   queries and keys of fused QKV rows: an RMS norm of each head if the model has one, then the rotation by position
  prompt   causal attention over prompts packed one behind the other, grouped heads
  store    keys and values of new tokens into a paged cache of 8-bit codes, a scale for each block of 16 tokens and head,
           and the blocks that they went into read back, as the values that the cache stands for
  cached   attention of new tokens over that cache: generation, a few drafted tokens, the next chunk of a long prompt

Rows are new with every seed; the cache, the tables of its pages and the output buffers are what such a program keeps. Head counts
are those of the benchmark's layers (64 heads over 8, 40, 32 of dimension 128) and generic ones.
"""
import math
import random

import torch

own = False

BLOCK = 16                               # tokens that share a scale
EPS = 1e-5
MOST_PAIRS = 64 * 16384 * 16384 // 2     # heads times pairs of tokens of a drawn prompt case: the largest listed one's
MOST_CACHED = 8 * 131072 * 128           # elements of keys of a drawn cached case
MOST_ROTATED = 4096 * 72 * 128


def listed():
    return [
        # token generation, one request: LLaMA-2-70B's fused QKV
        dict(name="rotate 1 token", kind="rotate", M=1, heads=64, kv=8, D=128, rot=128, interleaved=False, norm=False, far=4096),
        # a ragged batch far into long documents: norms, half of each head rotated, neighbours as pairs, small heads
        dict(name="rotate 333 tokens", kind="rotate", M=333, heads=24, kv=6, D=64, rot=32, interleaved=True, norm=True, far=1000000),
        # prefill, 70B's heads with norms
        dict(name="rotate 4096 tokens", kind="rotate", M=4096, heads=64, kv=8, D=128, rot=128, interleaved=False, norm=True, far=8192),
        # the shortest prompt, LLaMA-2-7B's heads
        dict(name="prompt 7 tokens", kind="prompt", M=7, S=1, heads=32, kv=32, D=128),
        # prompts of many lengths side by side, some of one token, one empty, small grouped heads
        dict(name="prompt 3001 tokens packed", kind="prompt", M=3001, S=9, heads=24, kv=6, D=64),
        # the largest: one long prompt, 70B's heads
        dict(name="prompt 16384 tokens", kind="prompt", M=16384, S=1, heads=64, kv=8, D=128),
        # batched generation: one token each of 32 sequences, anywhere in a block
        dict(name="store 32 tokens", kind="store", S=32, new=1, context=4096, kv=8, D=128, page=64),
        # prefill of a ragged batch, LLaMA-2-13B's heads, some behind a cached prefix
        dict(name="store 5 prompts", kind="store", S=5, new=1500, context=4000, kv=40, D=128, page=128),
        # token generation, one request of moderate length, 7B's heads, each with keys of its own
        dict(name="cached 1 sequence", kind="cached", S=1, new=1, context=1100, heads=32, kv=32, D=128, page=16),
        # batched generation: 48 sequences of many lengths, 70B's heads
        dict(name="cached 48 sequences", kind="cached", S=48, new=1, context=8192, heads=64, kv=8, D=128, page=64),
        # one very long document, a few drafted tokens
        dict(name="cached 131072 tokens", kind="cached", S=1, new=4, context=131072, heads=64, kv=8, D=128, page=128),
        # the next chunks of three long prompts, small heads, five to a key
        dict(name="cached chunks", kind="cached", S=3, new=400, context=9000, heads=30, kv=6, D=64, page=32),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def _heads(rng):
    kv = rng.choice([1, 2, 4, 5, 8, 8, 12, 32, 40])
    return kv * rng.choice([1, 2, 4, 5, 8] if kv <= 8 else [1, 2]), kv


def draw(rng):
    kind = rng.choice(["rotate", "prompt", "store", "cached", "cached"])
    while True:
        heads, kv = _heads(rng)
        D = rng.choice([64, 128, 128])
        if kind == "rotate":
            c = dict(kind=kind, M=_log_int(rng, 1, 16384), heads=heads, kv=kv, D=D, rot=rng.choice([D, D, D // 2, D // 4]),
                     interleaved=rng.random() < 0.4, norm=rng.random() < 0.5, far=rng.choice([4096, 1000000]))
            if c["M"] * (heads + kv) * D <= MOST_ROTATED:
                return c
        elif kind == "prompt":
            c = dict(kind=kind, M=_log_int(rng, 1, 16384), S=rng.choice([1, 1, _log_int(rng, 2, 64)]), heads=heads, kv=kv, D=D)
            if heads * sum(n * (n + 1) // 2 for n in _prompts(c)) <= MOST_PAIRS:
                return c
        else:
            c = dict(kind=kind, S=_log_int(rng, 1, 64), new=rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 9, 2000)]),
                     context=_log_int(rng, 17, 131072), kv=kv, D=D, page=rng.choice([16, 32, 64, 128]))
            if kind == "store":
                c["context"] = min(c["context"], 16384)
            else:
                c["heads"] = heads
            new, lengths = _batch(c)
            cached, M = sum(lengths) * kv * D, sum(new)
            pairs = heads * D * sum(n * l for n, l in zip(new, lengths))
            if cached <= MOST_CACHED and M * heads * D <= MOST_ROTATED and pairs <= MOST_PAIRS * 128 // 8:
                return c


def _prompts(c):
    """The lengths of a prompt case's sequences: M tokens in S parts of any length, every fifth part empty or one token."""
    rng = random.Random(c["M"] * 1009 + c["S"])
    cuts = sorted(rng.randint(0, c["M"]) for _ in range(c["S"] - 1))
    for i in range(4, len(cuts), 5):
        cuts[i] = min(c["M"], cuts[i - 1] + i % 2)
    cuts = sorted(cuts)
    return [b - a for a, b in zip([0] + cuts, cuts + [c["M"]])]


def _batch(c):
    """New tokens of each sequence and its length with them: the first has the whole context, the others any part of it."""
    rng = random.Random(c["context"] * 1009 + c["S"] * 31 + c["new"])
    new = [c["new"] if c["new"] <= 8 or i == 0 else rng.randint(1, c["new"]) for i in range(c["S"])]
    new = [min(n, c["context"]) for n in new]
    return new, [c["context"] if i == 0 else rng.randint(n, c["context"]) for i, n in enumerate(new)]


# ---- inputs, from the seed alone ---------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _keys(g, rows, kv, D):
    """Keys: some channels of each head are several times as large as the rest."""
    loud = 1.0 + 4.0 * (torch.rand((kv, D), generator=g, device="cuda") < 0.04)
    return (_randn(g, rows, kv, D) * loud).view(rows, kv * D).half()


def _starts(parts):
    return torch.tensor([0] + parts, dtype=torch.int32).cumsum(0).int().cuda()


def prepare(case, seed):
    c, g = case, _generator(seed)
    D, kv = c["D"], c["kv"]
    if c["kind"] == "rotate":
        M, heads = c["M"], c["heads"]
        runs = torch.randint(0, c["far"], (-(-M // 50),), generator=g, device="cuda")
        positions = (runs.repeat_interleave(50)[:M] + torch.arange(M, device="cuda") % 50).int()
        freq = 10000.0 ** (-torch.arange(0, c["rot"], 2, device="cuda").float() / c["rot"])
        return dict(case=c, qkv=_randn(g, M, (heads + 2 * kv) * D).half(), positions=positions, freq=freq,
                    gamma_q=(1.0 + 0.2 * _randn(g, D)).half() if c["norm"] else None,
                    gamma_k=(1.0 + 0.2 * _randn(g, D)).half() if c["norm"] else None,
                    out=torch.empty((M, (heads + kv) * D), dtype=torch.float16, device="cuda"))
    if c["kind"] == "prompt":
        M, heads = c["M"], c["heads"]
        parts = _prompts(c)
        # queries and keys as the rotation leaves them, values as the projection does
        rotated = torch.cat([(1.5 * _randn(g, M, heads * D)).half(), _keys(g, M, kv, D)], 1)
        qkv = _randn(g, M, (heads + 2 * kv) * D).half()
        return dict(case=c, parts=parts, q=rotated[:, :heads * D], k=rotated[:, heads * D:], v=qkv[:, (heads + kv) * D:],
                    starts=_starts(parts), out=torch.empty((M, heads * D), dtype=torch.float16, device="cuda"))
    new, lengths = _batch(c)
    S, page, M = c["S"], c["page"], sum(new)
    per = -(-max(lengths) // page)
    pages = sum(-(-n // page) for n in lengths)
    table = torch.full((S, per), -1, dtype=torch.int32)
    free = list(range(pages))
    random.Random(seed).shuffle(free)
    for s, n in enumerate(lengths):
        for i in range(-(-n // page)):
            table[s, i] = free.pop()
    slots = torch.randperm(S, generator=torch.Generator().manual_seed(seed)).int()
    s = dict(case=c, new=new, lengths=lengths, starts=_starts(new), table=table.cuda(), lengths_dev=torch.tensor(lengths, dtype=torch.int32).cuda(),
             slots=slots.cuda(), slots_host=slots.tolist())
    old = [n - m for n, m in zip(lengths, new)]
    whole = lengths if c["kind"] == "cached" else old        # what the cache holds before the pass
    k, v = _keys(g, sum(whole), kv, D), _randn(g, sum(whole), kv * D).half()
    if c["kind"] == "store":
        s["k"], s["v"] = _keys(g, M, kv, D), _randn(g, M, kv * D).half()
        s["touched"] = [m + n % BLOCK for m, n in zip(new, old)]        # tokens from the first new one's block on
        s["back"] = tuple(torch.empty((sum(s["touched"]), kv * D), dtype=torch.float16, device="cuda") for _ in range(2))
    else:
        s["q"] = (1.5 * _randn(g, M, c["heads"] * D)).half()
        s["out"] = torch.empty((M, c["heads"] * D), dtype=torch.float16, device="cuda")
    if own:
        import paper_2508_04405_amd as fq
        s["cache"] = fq.Cache(pages, page, kv, D, S)
        s["seqs"] = fq.Sequences(s["starts"], s["lengths_dev"], s["table"], s["slots"])
        if c["kind"] == "store":
            s["blocks"] = fq.Sequences(_starts(s["touched"]), s["lengths_dev"], s["table"], s["slots"])
        if sum(whole):
            fq.cache_append(s["cache"], k, v, fq.Sequences(_starts(whole), torch.tensor(whole, dtype=torch.int32).cuda(), s["table"], s["slots"]))
        if c["kind"] == "store" and c["new"] > BLOCK:    # (fewer leave the tokens before them where they are)
            s["before"] = s["cache"].recent.clone()
    else:
        s["codes"] = torch.zeros((2, pages * (page // BLOCK), kv, BLOCK, D), dtype=torch.int8, device="cuda")
        s["scales"] = torch.zeros((2, pages * (page // BLOCK), kv), dtype=torch.float16, device="cuda")
        s["recent"] = torch.zeros((2, S, BLOCK, kv, D), dtype=torch.float16, device="cuda")
        _fill(s, k, v, whole)
    return s


def _blocks(s, i, first, last):
    """Where blocks first .. last - 1 of sequence i lie in the plain cache."""
    per = s["case"]["page"] // BLOCK
    b = torch.arange(first, last, device="cuda")
    return s["table"][i].long()[b // per] * per + b % per


def _quantised(x):
    """Codes and scales of blocks [n, kv, 16, D]: one scale each, in 16 bits; a quotient in 32 bits rounded to the nearest code."""
    x = x.float()
    top = x.abs().amax((2, 3))
    scale = (top / 127.0).half()
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    return torch.round(x / scale.float()[:, :, None, None]).clamp(-128, 127).to(torch.int8), scale


def _put(s, i, which, rows, first):
    """Tokens rows [n, kv, D] of sequence i from position `first`, the beginning of a block, on."""
    n, kv, D = rows.shape
    done = n // BLOCK
    if done:
        at = _blocks(s, i, first // BLOCK, first // BLOCK + done)
        s["codes"][which, at], s["scales"][which, at] = _quantised(rows[:done * BLOCK].view(done, BLOCK, kv, D).transpose(1, 2))
    if n > done * BLOCK:
        s["recent"][which, s["slots_host"][i], :n - done * BLOCK] = rows[done * BLOCK:]


def _fill(s, k, v, lengths):
    c, at = s["case"], 0
    for i, n in enumerate(lengths):
        if n:
            for which, x in enumerate((k, v)):
                _put(s, i, which, x[at:at + n].view(n, c["kv"], c["D"]), 0)
        at += n
    if c["kind"] == "store":             # a pass finds the unfinished blocks as they were before it
        s["before"] = s["recent"].clone()


def _values(s, i, which, first, last):
    """Tokens first .. last - 1 of sequence i, whose length is `last`, as the cache stands for them: fp32 [n, kv, D]."""
    c = s["case"]
    b0, b1 = first // BLOCK, last // BLOCK
    at = _blocks(s, i, b0, max(b0, b1))
    x = s["codes"][which, at].float() * s["scales"][which, at].float()[:, :, None, None]
    x = x.transpose(1, 2).reshape(-1, c["kv"], c["D"])
    if last % BLOCK:
        x = torch.cat([x, s["recent"][which, s["slots_host"][i], :last % BLOCK].float()])
    return x[first - b0 * BLOCK:]


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if own:
        import paper_2508_04405_amd as fq
        if c["kind"] == "rotate":
            return fq.rotate_heads(s["qkv"], c["heads"], c["kv"], c["D"], s["positions"], s["freq"], gamma_q=s["gamma_q"],
                                   gamma_k=s["gamma_k"], eps=EPS, interleaved=c["interleaved"], out=s["out"])
        if c["kind"] == "prompt":
            return fq.prompt_attention(s["q"], s["k"], s["v"], c["heads"], c["kv"], s["starts"], out=s["out"])
        if c["kind"] == "store":
            if "before" in s:
                s["cache"].recent.copy_(s["before"])
            fq.cache_append(s["cache"], s["k"], s["v"], s["seqs"])
            return fq.cache_read(s["cache"], s["blocks"], out=s["back"])
        return fq.cache_attention(s["cache"], s["q"], c["heads"], s["seqs"], out=s["out"])
    return dict(rotate=_rotate, prompt=_prompt, store=_store, cached=_cached)[c["kind"]](s, c)


def _rotate(s, c):
    M, D, rot, all_heads = c["M"], c["D"], c["rot"], c["heads"] + c["kv"]
    x = s["qkv"][:, :all_heads * D].float().view(M, all_heads, D)
    if c["norm"]:
        gamma = torch.cat([s["gamma_q"].float().expand(c["heads"], D), s["gamma_k"].float().expand(c["kv"], D)])
        x = x / torch.sqrt(x.square().mean(2, keepdim=True) + EPS) * gamma
    angle = s["positions"].double()[:, None] * s["freq"].double()            # far positions: 32 bits lose the turns
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    y = x.clone()
    if c["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    s["out"].copy_(y.view(M, all_heads * D))
    return s["out"]


def _attend(q, k, v, first):
    """Grouped heads: q [n, heads, D], k and v [L, kv, D], all fp32; query i is token first + i and sees the keys up to itself."""
    n, heads, D = q.shape
    L, kv = k.shape[:2]
    group, out = heads // kv, torch.empty_like(q)
    see = first + torch.arange(n, device=q.device)
    for h in range(kv):
        for i in range(0, n, 2048):
            rows = q[i:i + 2048, h * group:(h + 1) * group]
            m, reach = rows.shape[0], min(L, first + i + 2048)
            score = (rows.reshape(m * group, D) @ k[:reach, h].t()).view(m, group, reach) / math.sqrt(D)
            score.masked_fill_((torch.arange(reach, device=q.device)[None, :] > see[i:i + m, None])[:, None], float("-inf"))
            score = torch.exp(score - score.amax(2, keepdim=True))
            total = score.sum(2, keepdim=True)
            out[i:i + m, h * group:(h + 1) * group] = (score.view(m * group, reach) @ v[:reach, h]).view(m, group, D) / total
    return out


def _prompt(s, c):
    D, at = c["D"], 0
    for n in s["parts"]:
        if n:
            q, k, v = (s[x][at:at + n].float().view(n, h, D) for x, h in (("q", c["heads"]), ("k", c["kv"]), ("v", c["kv"])))
            s["out"][at:at + n] = _attend(q, k, v, 0).view(n, -1)
        at += n
    return s["out"]


def _store(s, c):
    kv, D, at, to = c["kv"], c["D"], 0, 0
    s["recent"].copy_(s["before"])
    for i, (n, m, length) in enumerate(zip(s["new"], s["touched"], s["lengths"])):
        first = length - n
        begin = first // BLOCK * BLOCK
        for which, x in enumerate((s["k"], s["v"])):
            rows = torch.cat([s["recent"][which, s["slots_host"][i], :first - begin], x[at:at + n].view(n, kv, D)])
            _put(s, i, which, rows, begin)
            s["back"][which][to:to + m] = _values(s, i, which, begin, length).reshape(m, kv * D)
        at, to = at + n, to + m
    return s["back"]


def _cached(s, c):
    at = 0
    for i, (n, length) in enumerate(zip(s["new"], s["lengths"])):
        q = s["q"][at:at + n].float().view(n, c["heads"], c["D"])
        s["out"][at:at + n] = _attend(q, _values(s, i, 0, 0, length), _values(s, i, 1, 0, length), length - n).view(n, -1)
        at += n
    return s["out"]


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    c = case
    D, kv = c["D"], c["kv"]
    if c["kind"] == "rotate":
        elements = c["M"] * (c["heads"] + kv) * D
        return dict(bytes=4.0 * elements + 4.0 * c["M"] + 2.0 * c["rot"], flops=(9.0 if c["norm"] else 3.0) * elements)
    if c["kind"] == "prompt":
        return dict(bytes=4.0 * c["M"] * (c["heads"] + kv) * D, flops=4.0 * D * c["heads"] * sum(n * (n + 1) / 2 for n in _prompts(c)))
    new, lengths = _batch(c)
    if c["kind"] == "store":             # rows in, codes out; codes in, rows out
        touched = sum(new) + sum((length - n) % BLOCK for n, length in zip(new, lengths))
        return dict(bytes=(6.0 * sum(new) + 6.0 * touched) * kv * D, flops=6.0 * touched * kv * D)
    pairs = sum(n * (length - n) + n * (n + 1) / 2 for n, length in zip(new, lengths))
    return dict(bytes=sum(lengths) * kv * (2.0 * D + 0.25) + 4.0 * sum(new) * c["heads"] * D, flops=4.0 * D * c["heads"] * pairs)


# ---- the same in 64 bits -----------------------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False                # the inputs alone, no cache of the package's
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return dict(rotate=_rotate_exact, prompt=_prompt_exact, store=_store_exact, cached=_cached_exact)[case["kind"]](s, case)


def _rotate_exact(s, c):
    M, D, rot, heads = c["M"], c["D"], c["rot"], c["heads"]
    half, out = rot // 2, []
    turn = torch.exp(1j * (s["positions"].double()[:, None] * s["freq"].double()[None, :]))       # [M, rot / 2]
    for h in range(heads + c["kv"]):
        x = s["qkv"][:, h * D:(h + 1) * D].double()
        if c["norm"]:
            gamma = (s["gamma_q"] if h < heads else s["gamma_k"]).double()
            x = x * gamma * (x.pow(2).sum(1, keepdim=True) / D + EPS).pow(-0.5)
        pairs = torch.arange(rot, device=x.device)
        pairs = pairs.view(half, 2).t() if c["interleaved"] else pairs.view(2, half)
        z = torch.complex(x[:, pairs[0]], x[:, pairs[1]]) * turn
        x[:, pairs[0]], x[:, pairs[1]] = z.real, z.imag
        out.append(x)
    return torch.cat(out, 1)


def _softmax_exact(q, k, v, first):
    """One head, 64 bits: q [n, D], k and v [L, D]."""
    n, D = q.shape
    out = torch.empty_like(q)
    for i in range(0, n, 1024):
        reach = min(k.shape[0], first + i + 1024)
        score = q[i:i + 1024] @ k[:reach].t() * D ** -0.5
        ahead = torch.arange(reach, device=q.device) - torch.arange(first + i, first + i + score.shape[0], device=q.device)[:, None]
        out[i:i + 1024] = torch.softmax(torch.where(ahead > 0, -math.inf, score), 1) @ v[:reach]
    return out


def _heads_exact(q, k, v, c, first):
    D, group = c["D"], c["heads"] // c["kv"]
    part = lambda x, h: x[:, h * D:(h + 1) * D].double()
    return torch.cat([_softmax_exact(part(q, h), part(k, h // group), part(v, h // group), first) for h in range(c["heads"])], 1)


def _prompt_exact(s, c):
    out, at = [], 0
    for n in s["parts"]:
        rows = slice(at, at + n)
        out.append(_heads_exact(s["q"][rows], s["k"][rows], s["v"][rows], c, 0))
        at += n
    return torch.cat(out)


def _whole(s, i, which, length):
    """All tokens of sequence i in 64 bits, [length, kv * D], from the codes, block by block."""
    c = s["case"]
    kv, D, per, out = c["kv"], c["D"], c["page"] // BLOCK, []
    pages = s["table"][i].tolist()
    for p in range(-(-(length // BLOCK) // per)):
        last = min(per, length // BLOCK - p * per)
        at = slice(pages[p] * per, pages[p] * per + last)
        x = s["codes"][which, at].double() * s["scales"][which, at].double()[:, :, None, None]
        out.append(x.permute(0, 2, 1, 3).reshape(last * BLOCK, kv * D))
    out.append(s["recent"][which, s["slots_host"][i], :length % BLOCK].double().view(-1, kv * D))
    return torch.cat(out)


def _cached_exact(s, c):
    out, at = [], 0
    for i, (n, length) in enumerate(zip(s["new"], s["lengths"])):
        out.append(_heads_exact(s["q"][at:at + n], _whole(s, i, 0, length), _whole(s, i, 1, length), c, length - n))
        at += n
    return torch.cat(out)


def _store_exact(s, c):
    kv, D, out = c["kv"], c["D"], ([], [])
    for which, x in enumerate((s["k"], s["v"])):
        at = 0
        for i, (n, length) in enumerate(zip(s["new"], s["lengths"])):
            first = length - n
            older = s["before"][which, s["slots_host"][i], :first % BLOCK].double().view(-1, kv * D)
            rows = torch.cat([older, x[at:at + n].double()])
            for b in range(0, rows.shape[0] // BLOCK * BLOCK, BLOCK):
                block = rows[b:b + BLOCK].view(BLOCK, kv, D)
                scale = (block.abs().amax((0, 2), keepdim=True) / 127.0).half().double()
                scale[scale == 0] = 1.0
                rows[b:b + BLOCK] = (torch.round(block / scale).clamp(-128, 127) * scale).view(BLOCK, kv * D)
            out[which].append(rows)
            at += n
    return torch.cat(out[0]), torch.cat(out[1])
