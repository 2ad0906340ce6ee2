"""Batches whose rows choose their own weights: routing to experts, the experts' linear layers, low-rank adapters.

Three kinds of work, as a program that serves such a model calls them:

  route     scores of the experts, the k that each token goes to, their weights, and the tokens' rows grouped by expert
  experts   one linear layer of packed 6-bit experts on the rows grouped so: into the feed-forward width ("up"), or out of
            it with the weighted sum over each token's experts ("down")
  adapters  the low-rank adapters of many requests, added to the outputs of a projection that all of them share

Weights, scales, grouping and output buffers are what such a program keeps; activations are new with every seed. Hidden
sizes and widths are those of the benchmark's layers and generic ones.
"""
import math

import torch

own = False

MOST_MACS = 8192 * 22016 * 4096          # per pass of a drawn case: the largest listed one's
MOST_WEIGHTS = 8 * 22016 * 4096
MOST_ADAPTER = 4096 * (4096 + 12288)     # tokens times elements of the rows read and added to
NO_EXPERT = float("-inf")


def listed():
    return [
        # token generation, one request: eight experts, two a token, softmax over the chosen
        dict(name="route 1 token of 8", kind="route", M=1, E=8, k=2, score="softmax", bias=False, groups=1, top_groups=1,
             group_top=1, renormalise=True, scale=1.0, half=False, masked=0.0),
        # a short prompt, nothing a power of two: fp16 scores, weights as they are, a few experts and tokens masked
        dict(name="route 333 tokens of 60", kind="route", M=333, E=60, k=5, score="softmax", bias=False, groups=1, top_groups=1,
             group_top=1, renormalise=False, scale=1.0, half=True, masked=0.1),
        # prefill of a model of many experts: sigmoid scores, a bias for balance, four of eight groups
        dict(name="route 8192 tokens of 256", kind="route", M=8192, E=256, k=8, score="sigmoid", bias=True, groups=8, top_groups=4,
             group_top=2, renormalise=True, scale=2.5, half=False, masked=0.0),
        # token generation, one request: the fused gate|up layers of the six experts it goes to
        dict(name="experts up 1 token", kind="experts", side="up", M=1, E=64, k=6, H=2048, F=1408, bits=6, group=0, dropped=0.0),
        # batched decode: the down layers of eight wide experts at 24 requests, and their weighted sum
        dict(name="experts down 24 tokens", kind="experts", side="down", M=24, E=8, k=2, H=4096, F=11008, bits=8, group=0, dropped=0.0),
        # a ragged prompt with padding tokens, group-128 weight scales, widths that are no multiple of a tile
        dict(name="experts up 333 tokens g128", kind="experts", side="up", M=333, E=20, k=3, H=2176, F=1712, bits=8, group=128,
             dropped=0.1),
        # prefill through many small experts: the down layers and the weighted sum
        dict(name="experts down 2048 tokens", kind="experts", side="down", M=2048, E=64, k=6, H=2048, F=1408, bits=8, group=0,
             dropped=0.0),
        # the largest: prefill through eight wide experts
        dict(name="experts up 4096 tokens", kind="experts", side="up", M=4096, E=8, k=2, H=4096, F=11008, bits=6, group=0, dropped=0.0),
        # token generation, one request with an adapter on LLaMA-2-7B's attention output projection
        dict(name="adapters 1 token", kind="adapters", M=1, K=4096, N=4096, L=8, R=16, run=1, without=0.0),
        # batched decode: 48 requests with 32 adapters among them, some with none, on 70B's fused QKV
        dict(name="adapters 48 tokens", kind="adapters", M=48, K=8192, N=10240, L=32, R=64, run=1, without=0.2),
        # a mixed batch of prompts at odd lengths on widths that are no multiple of a tile
        dict(name="adapters 333 tokens", kind="adapters", M=333, K=5248, N=13664, L=5, R=32, run=71, without=0.2),
        # prefill of several prompts, LLaMA-2-7B's fused QKV
        dict(name="adapters 4096 tokens", kind="adapters", M=4096, K=4096, N=12288, L=6, R=16, run=700, without=0.1),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    kind = rng.choice(["route", "experts", "experts", "adapters"])
    while True:
        if kind == "route":
            groups = rng.choice([1, 1, 2, 4, 8])
            E = groups * _log_int(rng, max(2, 8 // groups), 256 // groups)
            top_groups = rng.randint(1, groups)
            k = rng.randint(1, min(8, E // groups * top_groups))
            return dict(kind=kind, M=_log_int(rng, 1, 8192), E=E, k=k, score=rng.choice(["softmax", "sigmoid"]),
                        bias=rng.random() < 0.5, groups=groups, top_groups=top_groups, group_top=rng.choice([1, 2]),
                        renormalise=rng.random() < 0.7, scale=rng.choice([1.0, 2.5]), half=rng.random() < 0.3,
                        masked=rng.choice([0.0, 0.0, 0.1]))
        if kind == "experts":
            E = _log_int(rng, 4, 128)
            c = dict(kind=kind, side=rng.choice(["up", "down"]), M=_log_int(rng, 1, 4096), E=E, k=rng.randint(1, min(8, E)),
                     H=128 * _log_int(rng, 4, 48), F=128 * _log_int(rng, 4, 96), bits=rng.choice([6, 8]),
                     group=rng.choice([0, 0, 128]), dropped=rng.choice([0.0, 0.0, 0.1]))
            if c["side"] == "up" and rng.random() < 0.3:
                c["F"] += 16 * rng.randint(1, 7)
            K, N = _layer(c)
            if E * K * N <= MOST_WEIGHTS and c["M"] * c["k"] * K * N <= MOST_MACS * (0.3 if c["group"] else 1.0):
                return c
        else:
            M = _log_int(rng, 1, 4096)
            c = dict(kind=kind, M=M, K=128 * _log_int(rng, 8, 224), N=32 * _log_int(rng, 16, 896), L=_log_int(rng, 1, 32),
                     R=rng.choice([16, 32, 64, 128]), run=rng.choice([1, 1 + M // 5]), without=rng.choice([0.0, 0.2]))
            if M * (c["K"] + c["N"]) * c["R"] // 16 <= MOST_ADAPTER and c["L"] * c["R"] * (c["K"] + c["N"]) <= 1 << 26:
                return c


def _layer(c):
    """(K, N) of an experts case."""
    return (c["H"], 2 * c["F"]) if c["side"] == "up" else (c["F"], c["H"])


# ---- inputs, from the seed alone ---------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device="cuda")


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _grouped(ids, count):
    """Rows of ids (flat) in the order of the id and then of the row, those with an id of -1 last; where each id's begin."""
    ids = ids.reshape(-1).long()
    key = torch.where(ids < 0, count, ids)
    order = torch.sort(key, stable=True)[1]
    sizes = torch.bincount(key, minlength=count + 1)[:count]
    offsets = torch.cat([sizes.new_zeros(1), sizes.cumsum(0)])
    return order.int(), offsets.int()


def _pack(codes, scales, group):
    """The packed form of int8 codes [E,N,K]: 3 KiB tiles of 32 rows x 128 k in which the last 32 k lie in the low bits
    of the other 96, then the scales (by tile for scales of groups), each expert's padded to 256 bytes."""
    E, N, K = codes.shape
    c = codes.view(E, N // 32, 32, K // 128, 4, 2, 16).permute(0, 1, 3, 4, 5, 2, 6) & 63
    tail = c[:, :, :, 3]
    planes = [((c[:, :, :, j] << 2) | ((tail >> (4 - 2 * j)) & 3)).to(torch.int8) for j in range(3)]
    tiles = torch.stack(planes, 3).reshape(E, -1).view(torch.uint8)
    s = scales if group == 0 else scales.view(E, N // 32, 32, K // 128).transpose(2, 3)
    s = s.contiguous().view(E, -1).view(torch.uint8)
    size = tiles.shape[1] + s.shape[1]
    return torch.cat([tiles, s, tiles.new_zeros((E, -size % 256))], 1)


def prepare(case, seed):
    c, g = case, _generator(seed)
    if c["kind"] == "route":
        M, E = c["M"], c["E"]
        logits = 1.5 * _randn(g, M, E) + 0.5 * _randn(g, E)
        if c["masked"]:        # experts that are away, and padding tokens
            logits[:, _rand(g, E) < c["masked"]] = NO_EXPERT
            logits[_rand(g, M) < c["masked"]] = NO_EXPERT
        return dict(case=c, logits=logits.half() if c["half"] else logits, bias=0.1 * _randn(g, E) if c["bias"] else None)
    if c["kind"] == "experts":
        M, E, k = c["M"], c["E"], c["k"]
        K, N = _layer(c)
        scores = _randn(g, M, E) + 0.3 * _randn(g, E)
        weights, experts = torch.topk(scores.softmax(1), k, 1)
        weights /= weights.sum(1, keepdim=True)
        experts = experts.int()
        if c["dropped"]:
            gone = _rand(g, M) < c["dropped"]
            experts[gone], weights[gone] = -1, 0.0
        order, offsets = _grouped(experts, E)
        codes = torch.empty((E, N, K), dtype=torch.int8, device="cuda")
        for e in range(E):
            codes[e] = _randn(g, N, K).mul_(9.0).round_().clamp_(-32, 31)
        rows = M if c["side"] == "up" else M * k
        most = 31 if c["bits"] == 6 else 127
        xq = _randn(g, rows, K).mul_(most / 4.0).round_().clamp_(-most, most).to(torch.int8)
        sx = (_rand(g, rows) + 0.5).mul_(4.0 / most).half()
        sw = (_rand(g, *((E, N) if c["group"] == 0 else (E, N, K // 128))) + 0.5).mul_(0.002).half()
        s = dict(case=c, codes=codes, sw=sw, packed=_pack(codes, sw, c["group"]), xq=xq, sx=sx, experts=experts, weights=weights,
                 order=order, offsets=offsets, rows=torch.zeros((M * k, N), dtype=torch.float16, device="cuda"))
        if c["side"] == "down":
            s["out"] = torch.empty((M, N), dtype=torch.float16, device="cuda")
        return s
    M, K, N, L, R = c["M"], c["K"], c["N"], c["L"], c["R"]
    runs = -(-M // c["run"])
    ids = torch.randint(0, L, (runs,), generator=g, device="cuda", dtype=torch.int32)
    ids[_rand(g, runs) < c["without"]] = -1
    ids = ids.repeat_interleave(c["run"])[:M].contiguous()
    order, offsets = _grouped(ids, L)
    x = _randn(g, M, K)
    x[:, torch.randperm(K, generator=g, device="cuda")[:max(1, K // 100)]] *= 20.0
    return dict(case=c, a=(_randn(g, L, R, K) / math.sqrt(K)).half(), b=(0.05 * _randn(g, L, N, R)).half(),
                scale=_rand(g, L) + 0.5, x=x.half(), y=_randn(g, M, N).half(), ids=ids, order=order, offsets=offsets,
                out=torch.empty((M, N), dtype=torch.float16, device="cuda"))


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if own:
        import paper_2508_04405_amd as fq
        if c["kind"] == "route":
            r = fq.route_experts(s["logits"], c["k"], score=c["score"], bias=s["bias"], groups=c["groups"],
                                 top_groups=c["top_groups"], group_top=c["group_top"], renormalise=c["renormalise"],
                                 scale=c["scale"])
            return dict(experts=r.experts, weights=r.weights, order=r.order, offsets=r.offsets)
        if c["kind"] == "experts":
            K, N = _layer(c)
            up = c["side"] == "up"
            y = fq.expert_linear(s["packed"], N, K, s["xq"], s["sx"], s["order"], s["offsets"], group=c["group"],
                                 k=c["k"] if up else 0, scatter=not up, out=s["rows"])
            return y if up else fq.combine_experts(y, s["experts"], s["weights"], out=s["out"])
        return fq.adapters(s["a"], s["b"], s["scale"], s["x"], s["order"], s["offsets"], s["y"], out=s["out"])
    return dict(route=_route, experts=_experts, adapters=_adapters)[c["kind"]](s, c)


def _best(values, count):
    """The indexes of the largest values of each row, ties to the lowest index, and whether they are above -inf."""
    at = torch.sort(values, dim=1, descending=True, stable=True)[1][:, :count]
    return at, values.gather(1, at) > NO_EXPERT


def _route(s, c):
    M, E, k, groups = c["M"], c["E"], c["k"], c["groups"]
    logits = s["logits"].double()            # choices between close scores are made in 64 bits
    there = logits > NO_EXPERT
    if c["score"] == "softmax":
        top = logits.amax(1, keepdim=True)
        e = torch.where(there, torch.exp(logits - torch.where(top > NO_EXPERT, top, 0.0)), 0.0)
        score = e / e.sum(1, keepdim=True).clamp_min(1e-300)
    else:
        score = torch.where(there, 1.0 / (1.0 + torch.exp(-logits)), 0.0)
    choice = torch.where(there, score + s["bias"].double() if s["bias"] is not None else score, NO_EXPERT)
    if groups > 1:
        members = choice.view(M, groups, E // groups)
        best = members.topk(min(c["group_top"], E // groups), dim=2)[0]
        of_group = torch.where(best[:, :, 0] > NO_EXPERT, torch.where(best > NO_EXPERT, best, 0.0).sum(2), NO_EXPERT)
        at, _ = _best(of_group, c["top_groups"])
        kept = torch.zeros((M, groups), dtype=torch.bool, device=logits.device).scatter_(1, at, True)
        choice = torch.where(kept[:, :, None], members, NO_EXPERT).view(M, E)
    at, valid = _best(choice, k)
    weights = torch.where(valid, score.gather(1, at), 0.0)
    if c["renormalise"]:
        total = weights.sum(1, keepdim=True)
        weights = torch.where(total > 0, weights / torch.where(total > 0, total, 1.0), 0.0)
    experts = torch.where(valid, at, -1).int()
    order, offsets = _grouped(experts, E)
    return dict(experts=experts, weights=(weights * c["scale"]).float(), order=order, offsets=offsets)


def _experts(s, c):
    K, N = _layer(c)
    up, E, k, group = c["side"] == "up", c["E"], c["k"], c["group"]
    order, offsets, out = s["order"], s["offsets"].long(), s["rows"]
    total = int(offsets[-1])
    order = order[:total].long()
    rows = torch.arange(total, device=order.device)
    of = torch.bucketize(rows, offsets[1:], right=True)                 # each row's expert
    source = order // k if up else rows
    x = s["xq"][source].float()
    if group:
        x = x * s["sx"][source].float()[:, None]
        scaled = lambda codes, sw: (codes.float().view(-1, N, K // 128, 128) * sw.float()[..., None]).view(-1, N, K)
    else:
        scaled = lambda codes, sw: codes.float()
    if total < E:                                                       # few rows: the weights of each
        y = torch.bmm(scaled(s["codes"][of], s["sw"][of]), x[:, :, None])[:, :, 0]
    else:                                                               # each expert's rows side by side
        most = int((offsets[1:] - offsets[:-1]).max())
        at = of * most + rows - offsets[of]
        side = x.new_zeros((E * most, K))
        side[at] = x
        y = torch.bmm(scaled(s["codes"], s["sw"]), side.view(E, most, K).transpose(1, 2).contiguous())
        y = y.transpose(1, 2).reshape(E * most, N)[at]
    if not group:
        y = y * (s["sx"][source].float()[:, None] * s["sw"][of].float())
    if up:
        out[:total] = y.half()
        return out
    out[order] = y.half()
    rows_of = torch.where((s["experts"] >= 0)[:, :, None], out.view(c["M"], k, N).float(), 0.0)
    s["out"].copy_((rows_of * s["weights"][:, :, None]).sum(1))
    return s["out"]


def _adapters(s, c):
    M, K, N, L, R = c["M"], c["K"], c["N"], c["L"], c["R"]
    mine = torch.arange(L, device=s["ids"].device)[None, :] == s["ids"][:, None]
    h = (s["x"].float() @ s["a"].view(L * R, K).float().t()).view(M, L, R)
    h = torch.where(mine[:, :, None], h * s["scale"][:, None], 0.0).view(M, L * R)
    s["out"].copy_(s["y"].float() + h @ s["b"].float().transpose(1, 2).reshape(L * R, N))
    return s["out"]


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    c = case
    M = c["M"]
    if c["kind"] == "route":
        E, k = c["E"], c["k"]
        return dict(bytes=M * E * (2.0 if c["half"] else 4.0) + 12.0 * M * k + 4.0 * (E + 1), flops=8.0 * M * E)
    if c["kind"] == "experts":
        K, N = _layer(c)
        E, k = c["E"], c["k"]
        rows = M * k
        touched = E * (1.0 - (1.0 - k / E) ** M)
        weights = touched * (0.75 * N * K + 2.0 * N * (K // 128 if c["group"] else 1))
        if c["side"] == "up":
            return dict(bytes=weights + M * (K + 2.0) + 4.0 * rows + 2.0 * rows * N, flops=2.0 * rows * K * N)
        return dict(bytes=weights + rows * (K + 10.0) + 2.0 * M * N, flops=2.0 * rows * K * N)
    K, N, L, R = c["K"], c["N"], c["L"], c["R"]
    runs = -(-M // c["run"]) * (1.0 - c["without"])
    used = L * (1.0 - (1.0 - 1.0 / L) ** runs)
    with_one = M * (1.0 - c["without"])
    return dict(bytes=2.0 * with_one * K + 4.0 * M * N + 2.0 * used * R * (K + N), flops=2.0 * with_one * R * (K + N))


# ---- the same in 64 bits -----------------------------------------------------------------------------------------

def exact(case, seed):
    c, s = case, prepare(case, seed)
    return dict(route=_route_exact, experts=_experts_exact, adapters=_adapters_exact)[c["kind"]](s, c)


def _route_exact(s, c):
    import numpy as np
    M, E, k = c["M"], c["E"], c["k"]
    logits = s["logits"].double().cpu().numpy()
    bias = s["bias"].double().cpu().numpy() if s["bias"] is not None else np.zeros(E)
    experts, weights = np.full((M, k), -1, dtype=np.int32), np.zeros((M, k))
    for m in range(M):
        row = logits[m]
        present = [e for e in range(E) if row[e] > -math.inf]
        if not present:
            continue
        if c["score"] == "softmax":
            p = np.exp(row - row.max())
            p = p / p.sum()
        else:
            p = 1.0 / (1.0 + np.exp(-row))
        choice = p + bias
        if c["groups"] > 1:
            size, value = E // c["groups"], {}
            for e in present:
                value.setdefault(e // size, []).append(choice[e])
            value = {q: sum(sorted(v)[-c["group_top"]:]) for q, v in value.items()}
            kept = sorted(value, key=lambda q: (-value[q], q))[:c["top_groups"]]
            present = [e for e in present if e // size in kept]
        present = sorted(present, key=lambda e: (-choice[e], e))[:k]
        w = p[present]
        if c["renormalise"] and w.sum() > 0:
            w = w / w.sum()
        experts[m, :len(present)], weights[m, :len(present)] = present, w * c["scale"]
    flat = experts.reshape(-1)
    by_expert = [np.flatnonzero(flat == e) for e in range(E)]
    order = np.concatenate(by_expert + [np.flatnonzero(flat < 0)]).astype(np.int32)
    offsets = np.cumsum([0] + [v.size for v in by_expert]).astype(np.int32)
    return dict(experts=experts, weights=weights, order=order, offsets=offsets)


def _experts_exact(s, c):
    K, N = _layer(c)
    up, k = c["side"] == "up", c["k"]
    out = torch.zeros((c["M"] * k, N), dtype=torch.float64, device="cuda")
    begins = s["offsets"].tolist()
    for e, (r0, r1) in enumerate(zip(begins, begins[1:])):
        if r0 == r1:
            continue
        slots = s["order"][r0:r1].long()
        at = torch.div(slots, k, rounding_mode="floor") if up else torch.arange(r0, r1, device="cuda")
        w = s["codes"][e].double()
        w = w * s["sw"][e].double().repeat_interleave(128, 1) if c["group"] else w * s["sw"][e].double()[:, None]
        y = (s["xq"][at].double() * s["sx"][at].double()[:, None]) @ w.t()
        if up:
            out[r0:r1] = y
        else:
            out[slots] = y
    if up:
        return out
    out = out.half().double().view(c["M"], k, N)           # the products' rows are fp16 by definition
    return (out * s["weights"].double()[:, :, None]).sum(1)


def _adapters_exact(s, c):
    out = s["y"].double()
    for i in range(c["L"]):
        rows = torch.nonzero(s["ids"] == i)[:, 0]
        if rows.numel():
            low = s["x"][rows].double() @ s["a"][i].double().t()
            out[rows] += s["scale"][i].double() * (low @ s["b"][i].double().t())
    return out
