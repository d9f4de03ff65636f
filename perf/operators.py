"""Timed cases of the 4-bit node states, decode over them, accumulated attention weights, and eviction by those weights.

Four operators that a serving loop runs side by side:

  store    a node's K/V put into 4 bits and read back (gf_node_kv4_write, gf_node_kv_read)
  decode   one decode step of one layer over paths whose nodes are held in 4 bits, in bf16, or some each
           (gf_path_attention_decode)
  weights  what share of the batch's attention every resident token received in that step, per KV head
           (gf_path_attention_weights)
  evict    a node's tokens with the largest accumulated weight become the state of another node
           (gf_node_kv_evict)

The 4-bit format.  Every 64 neighbouring entries of one token and KV head form a group with two bf16 numbers: lo, the group's
least value, and s, the bf16 nearest to (hi - lo) / 16.  An entry x has the code floor((x - lo) / s) held within 0 .. 15 (0 where
s is 0), and stands for lo + s (code + 1/2), the middle of its cell (for lo itself where s is 0).

Values follow the seed; lengths, paths and which nodes are held in 4 bits follow the case (its "layout")."""
import math
import random

import numpy as np
import torch

own = False

GROUP = 64


def listed():
    """What each stands for: a single new token (latency alone), an odd segment at the small head size, one long document; the tiny graph; a
    batch of agents over a shared prompt; one request over a very long context (few rows, work split along the tokens); the
    full-depth batch with a fixed token budget, a third of its nodes kept in bf16; the same batches' weights; a small node cut down, and
    the caches of several requests cut to a half."""
    return [
        dict(name="store-1", op="store", tokens=1, hkv=8, d=128),
        dict(name="store-577-d64", op="store", tokens=577, hkv=4, d=64),
        dict(name="store-32768", op="store", tokens=32768, hkv=8, d=128),
        dict(name="decode-tiny", op="decode", hq=4, hkv=4, d=64, requests=8, nodes=16, root=64, lo=16, hi=64, depth=4, suffix=16, skew=1.0,
             four=1.0, layout=1),
        dict(name="decode-batch", op="decode", hq=32, hkv=8, d=128, requests=256, nodes=256, root=2048, lo=128, hi=1024, depth=6, suffix=512,
             skew=1.0, four=1.0, layout=2),
        dict(name="decode-long", op="decode", hq=32, hkv=8, d=128, requests=1, nodes=5, root=32768, lo=8000, hi=8200, depth=5, suffix=100,
             skew=1.0, four=1.0, layout=3),
        dict(name="decode-mixed-large", op="decode", hq=32, hkv=8, d=128, requests=1024, nodes=1024, root=2048, lo=32, hi=600, depth=7, suffix=400,
             skew=1.5, four=0.67, layout=4),
        dict(name="weights-tiny-4bit", op="weights", hq=8, hkv=4, d=64, requests=8, nodes=16, root=64, lo=16, hi=64, depth=4, suffix=16, skew=1.0,
             four=1.0, layout=5, add=True),
        dict(name="weights-batch", op="weights", hq=32, hkv=8, d=128, requests=256, nodes=256, root=2048, lo=128, hi=1024, depth=6, suffix=512,
             skew=1.0, four=0.0, layout=6, add=False),
        dict(name="weights-shared", op="weights", hq=32, hkv=8, d=128, requests=512, nodes=200, root=8192, lo=64, hi=512, depth=6, suffix=256,
             skew=2.0, four=0.5, layout=7, add=False),
        dict(name="evict-300", op="evict", hkv=8, d=128, count=1, layers=1, lo=300, hi=300, keep=0.4, first=4, last=32, four=0.0, layout=8),
        dict(name="evict-4x8192", op="evict", hkv=8, d=128, count=4, layers=2, lo=6000, hi=8192, keep=0.5, first=4, last=256, four=0.5, layout=9),
    ]


def draw(rng):
    """One more case of the same ranges: token counts, batch sizes and lengths spread over their logarithms."""
    def between(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    op = rng.choice(["store", "decode", "decode", "weights", "weights", "evict"])
    hq, hkv, d = rng.choice([(32, 8, 128), (32, 8, 128), (4, 4, 64), (8, 4, 64), (16, 2, 128), (32, 4, 64)])
    layout = rng.randrange(1 << 20)
    if op == "store":
        return dict(op=op, tokens=between(1, 32768), hkv=hkv, d=d)
    if op == "evict":
        hi = between(2, 8192)
        return dict(op=op, hkv=hkv, d=d, count=rng.randint(1, 4), layers=rng.randint(1, 2), lo=max(1, hi // 2), hi=hi, keep=rng.choice([0.1, 0.5, 0.9]),
                    first=rng.choice([0, 4]), last=rng.choice([0, 1, 32]), four=rng.choice([0.0, 0.5, 1.0]), layout=layout)
    requests = between(1, 256)
    hi = between(16, 1024)
    case = dict(op=op, hq=hq, hkv=hkv, d=d, requests=requests, nodes=between(8, 256), root=between(1, 4096), lo=max(1, hi // 8), hi=hi,
                depth=rng.randint(2, 7), suffix=rng.choice([0, 63, 512]), skew=rng.choice([1.0, 2.0]), four=rng.choice([0.0, 0.5, 1.0]) if op == "weights" else
                rng.choice([0.5, 1.0, 1.0]), layout=layout)
    if op == "weights":
        case["add"] = rng.choice([True, False])
    return case


# ---- what a case consists of (from the case alone) ---------------------------------------------------------


def _structure(case):
    """Node lengths, every request's path, and which nodes are held in 4 bits.  Node 0 is the root of every path; the other
    shared nodes stand in levels, one node of each level on a path; a request's own suffix comes last.  One node in eight is empty."""
    rng = random.Random(case["layout"])
    if case["op"] == "evict":
        lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["count"])]
        four = [i + 1 <= case["four"] * case["count"] for i in range(case["count"])]
        keep = [max(case["first"] + case["last"], int(n * case["keep"])) for n in lens]
        return dict(lens=lens, four=four, keep=keep)
    n, levels = case["nodes"], case["depth"] - 1
    lens = [case["root"]] + [0 if i % 8 == 7 else rng.randint(case["lo"], case["hi"]) for i in range(1, n)]
    per = max(1, (n - 1) // max(1, levels))
    paths = []
    for r in range(case["requests"]):
        path = [0]
        for level in range(rng.randint(max(1, levels - 2), levels) if levels else 0):
            pick = 1 + level * per + int(per * rng.random() ** case["skew"])
            if pick < n:
                path.append(pick)
        lens.append(rng.randint(0, case["suffix"]))
        path.append(n + r)
        paths.append(path)
    four = [rng.random() < case["four"] for _ in lens]
    return dict(lens=lens, paths=paths, four=four)


def _used(st):
    """The nodes that are on a path and hold tokens, ascending."""
    return [v for v in sorted({v for p in st["paths"] for v in p}) if st["lens"][v] > 0]


def work(case):
    """Bytes that no implementation can do without, every input once and every output once, and the products' operations."""
    if case["op"] == "store":
        return dict(bytes=8 * case["tokens"] * case["hkv"] * case["d"], flops=6 * case["tokens"] * case["hkv"] * case["d"])
    st, hkv, d = _structure(case), case["hkv"], case["d"]
    row = {False: 2 * d, True: d // 2 + d // GROUP * 4}  # bytes of one token's K (or V) of one KV head
    if case["op"] == "evict":
        b = 0
        for n, four, keep in zip(st["lens"], st["four"], st["keep"]):
            m = min(n, keep)
            b += case["layers"] * hkv * (4 * n + m * (4 + 4 + 2 * row[four] + 4 * d))
        return dict(bytes=b, flops=case["layers"] * hkv * sum(st["lens"]))
    parts = 2 if case["op"] == "decode" else 1
    b = sum(st["lens"][v] * hkv * parts * row[st["four"][v]] for v in _used(st))
    ctx = sum(st["lens"][v] for p in st["paths"] for v in p)
    b += case["requests"] * case["hq"] * (2 * d + 4)  # queries and log-sum-exps
    if case["op"] == "decode":
        b += case["requests"] * case["hq"] * 2 * d
    else:
        b += sum(st["lens"][v] for v in _used(st)) * hkv * 4 * (2 if case["add"] else 1)
    return dict(bytes=b, flops=2 * parts * d * case["hq"] * ctx)


# ---- inputs --------------------------------------------------------------------------------------------


def _kv(gen, n, hkv, d):
    """Keys and values of n tokens, bf16: normal values, every channel with a spread of its own, a few keys' channels with a large one."""
    spread = torch.exp(0.5 * torch.randn(2, hkv, d, generator=gen, device="cuda"))
    spread[0, :, ::32] *= 3.0
    k = torch.randn(n, hkv, d, generator=gen, device="cuda").mul_(spread[0] * 0.6).to(torch.bfloat16)
    v = torch.randn(n, hkv, d, generator=gen, device="cuda").mul_(spread[1]).to(torch.bfloat16)
    return k, v


def _inputs(case, seed):
    """The tensors of a case, from the seed."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] == "store":
        k, v = _kv(gen, case["tokens"], case["hkv"], case["d"])
        return dict(k=k, v=v)
    st = _structure(case)
    if case["op"] == "evict":
        kv = [_kv(gen, n * case["layers"], case["hkv"], case["d"]) for n in st["lens"]]
        shape = [(case["layers"], n, case["hkv"], case["d"]) for n in st["lens"]]
        # weights summed over some steps: a few tokens carry much of them, many are equal (zero among them)
        w = [torch.floor(torch.rand(case["layers"], case["hkv"], n, generator=gen, device="cuda") ** 6 * 4096) / 256 for n in st["lens"]]
        return dict(st=st, k=[a.view(s) for (a, _), s in zip(kv, shape)], v=[b.view(s) for (_, b), s in zip(kv, shape)], w=w)
    # where every node's tokens stand: the nodes in bf16 first, then those in 4 bits, each from a multiple of 64 on
    used = sorted(_used(st), key=lambda u: (st["four"][u], u))
    ends = np.cumsum([-(-st["lens"][u] // 64) * 64 for u in used])
    start, total = dict(zip(used, [0] + ends.tolist())), int(ends[-1])
    k, v = _kv(gen, total, case["hkv"], case["d"])
    q = torch.randn(case["requests"], case["hq"], case["d"], generator=gen, device="cuda").to(torch.bfloat16)
    # every request's tokens as rows of k and v, padded with -1
    rows = [np.concatenate([np.arange(start[u], start[u] + st["lens"][u]) for u in p if st["lens"][u] > 0] or [np.zeros(0, np.int64)]) for p in st["paths"]]
    most = max(1, max(len(r) for r in rows))
    table = np.full((len(rows), most), -1, np.int64)
    for r, x in enumerate(rows):
        table[r, :len(x)] = x
    four = np.repeat([st["four"][u] for u in used], np.diff(ends, prepend=0))
    out = dict(st=st, used=used, start=start, k=k, v=v, q=q, table=torch.from_numpy(table).cuda(), four=torch.from_numpy(four).cuda())
    if case["op"] == "weights":
        out["before"] = torch.rand(case["hkv"], total, generator=gen, device="cuda")
    return out


def _pack(x):
    """The 4-bit form of x [..., d]: two codes a byte, and each group's s and lo in bf16."""
    y = x.float().unflatten(-1, (-1, GROUP))
    lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    s = (hi * 0.0625 - lo * 0.0625).to(torch.bfloat16)
    f = s.float()
    code = torch.where(f > 0, torch.floor((y * 0.0625 - lo * 0.0625) / f * 16.0), torch.zeros_like(y)).clamp(0, 15).to(torch.uint8).flatten(-2)
    return dict(code=code[..., 0::2] | (code[..., 1::2] << 4), s=s.squeeze(-1), lo=lo.to(torch.bfloat16).squeeze(-1))


def _unpack(p):
    """The values that a 4-bit form stands for, in 32 bits."""
    code = torch.stack([p["code"] & 15, p["code"] >> 4], -1).flatten(-2).float().unflatten(-1, (-1, GROUP))
    s = p["s"].float().unsqueeze(-1)
    return torch.where(s > 0, p["lo"].float().unsqueeze(-1) + s * (code + 0.5), p["lo"].float().unsqueeze(-1).expand_as(code)).flatten(-2)


def prepare(case, seed):
    x = _inputs(case, seed)
    state = dict(case=case, **x)
    if case["op"] == "store":
        if own:
            state["pa"] = _handle(case, [case["tokens"]], [[0]], [True])
        return state
    st = x["st"]
    if case["op"] == "evict":
        if own:
            n = case["count"]
            pa = _handle(case, st["lens"] + [min(a, b) for a, b in zip(st["lens"], st["keep"])], [[i] for i in range(2 * n)], st["four"] * 2)
            for i in range(n):
                for layer in range(case["layers"]):
                    pa.write_node(i, layer, x["k"][i][layer], x["v"][i][layer])
            state["pa"], state["weights"] = pa, pa.new_weights()
            for i in range(n):
                pa.node_weights(state["weights"], i).copy_(x["w"][i])
            torch.cuda.synchronize()
        else:
            state["k"] = [_pack(k) if f else k for k, f in zip(x["k"], st["four"])]
            state["v"] = [_pack(v) if f else v for v, f in zip(x["v"], st["four"])]
        return state
    if case["op"] == "weights":
        state["lse"] = _attend(x["q"], _held(x["k"], x["four"]), None, x["table"])[1]
    if own:
        pa = _handle(case, st["lens"], st["paths"], st["four"])
        for u in x["used"]:
            rows = slice(x["start"][u], x["start"][u] + st["lens"][u])
            pa.write_node(u, 0, x["k"][rows], x["v"][rows])
        pa.build()
        state["pa"] = pa
        if case["op"] == "weights":
            state["weights"] = pa.new_weights()
            first = pa.node_slot(x["used"][0])
            state["sums"] = state["weights"][0, :, first:first + x["k"].shape[0]]  # this layer's, in the order of the rows
        torch.cuda.synchronize()
        del state["k"], state["v"]
    else:
        state["k4"], state["v4"] = _pack(x["k"]), _pack(x["v"])
    return state


def _handle(case, lens, paths, four):
    """A wGraph handle for these nodes and paths (every node a request's own: no edges), pools sized to fit."""
    from paper_2605_22566_b200 import runtime, workloads
    w = workloads.Workload(name="operators", config_id=-1, seed=0, mode="decode", num_layers=case.get("layers", 1), num_q_heads=case.get("hq", case["hkv"]),
                           num_kv_heads=case["hkv"], head_dim=case["d"], num_shared_nodes=0, num_nodes=len(lens), edge_src=np.zeros(0, np.int32),
                           edge_dst=np.zeros(0, np.int32), node_len=np.array(lens, np.int32),
                           path_ptr=np.concatenate([[0], np.cumsum([len(p) for p in paths])]).astype(np.int32), path_node=np.array(sum(paths, []), np.int32))
    return runtime.PathAttention(w, kv4_nodes=[v for v, f in enumerate(four) if f])


# ---- the operators' plain forms --------------------------------------------------------------------------


def _held(k, four):
    """What the cache holds of k, in 32 bits: the rows in 4 bits as the values that they stand for."""
    return torch.where(four[:, None, None], _unpack(_pack(k)), k.float())


def _attend(q, k, v, table):
    """softmax(q k / sqrt(d)) v over every request's rows, its log-sum-exp, and what share each row received, [hkv, rows]; all in 32 bits.
    As many requests at a time as the gathered rows have room for."""
    hkv, d = k.shape[1:]
    qf = q.float().view(q.shape[0], hkv, -1, d) / math.sqrt(d)
    step = max(1, (1 << 29) // (table.shape[1] * hkv * d))
    out, lse = [], []
    for r in range(0, q.shape[0], step):
        t = table[r:r + step]
        s = torch.einsum("rhgd,rlhd->rhgl", qf[r:r + step], k[t.clamp(min=0)]).masked_fill(t[:, None, None] < 0, float("-inf"))
        m = s.amax(-1, keepdim=True).clamp(min=-3e38)
        p = torch.exp(s - m)
        total = p.sum(-1, keepdim=True)
        lse.append((m + torch.log(total)).squeeze(-1).flatten(1))
        if v is not None:
            out.append((torch.einsum("rhgl,rlhd->rhgd", p, v[t.clamp(min=0)]) / total.clamp(min=1e-38)).flatten(1, 2))
    return torch.cat(out) if out else None, torch.cat(lse)


def _shares(q, k, lse, table):
    """The sum over requests and query heads of exp(score - lse), for every row and KV head: [hkv, rows]."""
    hkv, d = k.shape[1:]
    qf = q.float().view(q.shape[0], hkv, -1, d) / math.sqrt(d)
    got = torch.zeros(k.shape[0], hkv, dtype=torch.float64, device=k.device)  # long sums
    step = max(1, (1 << 29) // (table.shape[1] * hkv * d))
    for r in range(0, q.shape[0], step):
        t = table[r:r + step]
        s = torch.einsum("rhgd,rlhd->rhgl", qf[r:r + step], k[t.clamp(min=0)]) - lse[r:r + step].view(t.shape[0], hkv, -1, 1)
        p = torch.exp(s).sum(2).masked_fill(t[:, None] < 0, 0.0)
        got.index_add_(0, t.clamp(min=0).flatten(), p.transpose(1, 2).flatten(0, 1).double())
    return got.t().float()


def _evict(k, v, w, keep, first, last):
    """The tokens kept per (layer, KV head), ascending: the first and last few, then those of the largest weight, ties to the lowest index."""
    n = w.shape[-1]
    m = min(n, keep)
    at = torch.arange(n, device=w.device)
    order = torch.sort(w.masked_fill((at < first) | (at >= n - last), float("inf")), dim=-1, descending=True, stable=True)[1]
    kept = torch.sort(order[..., :m], dim=-1)[0]
    rows = kept.transpose(1, 2).unsqueeze(-1)

    def pick(x):
        if isinstance(x, dict):
            return _unpack({name: torch.take_along_dim(y, rows, 1) for name, y in x.items()}).to(torch.bfloat16)
        return torch.take_along_dim(x, rows, 1)
    return dict(kept=kept.int(), k=pick(k), v=pick(v), w=torch.take_along_dim(w, kept, -1))


def run(state):
    case = state["case"]
    if own:
        return _run_own(state)
    if case["op"] == "store":
        return dict(k=_unpack(_pack(state["k"])).to(torch.bfloat16), v=_unpack(_pack(state["v"])).to(torch.bfloat16))
    if case["op"] == "evict":
        return [_evict(k, v, w, keep, case["first"], case["last"]) for k, v, w, keep in zip(state["k"], state["v"], state["w"], state["st"]["keep"])]
    four = state["four"][:, None, None]
    k = torch.where(four, _unpack(state["k4"]), state["k"].float())
    if case["op"] == "weights":
        got = _shares(state["q"], k, state["lse"], state["table"])
        return state["before"] + got if case["add"] else got
    out, lse = _attend(state["q"], k, torch.where(four, _unpack(state["v4"]), state["v"].float()), state["table"])
    return dict(out=out.to(torch.bfloat16), lse=lse)


def _run_own(state):
    case, pa = state["case"], state["pa"]
    if case["op"] == "store":
        pa.write_node(0, 0, state["k"], state["v"])
        k, v = pa.load_node(0, 0)
        return dict(k=k, v=v)
    if case["op"] == "evict":
        n = case["count"]
        kept = pa.evict([(n + i, i, state["st"]["keep"][i], case["first"], case["last"]) for i in range(n)], state["weights"])
        out = []
        for i in range(n):
            k, v = zip(*[pa.load_node(n + i, layer) for layer in range(case["layers"])])
            out.append(dict(kept=kept[i], k=torch.stack(k), v=torch.stack(v), w=pa.node_weights(state["weights"], n + i)))
        return out
    if case["op"] == "weights":
        if case["add"]:  # the sums of the steps before this one
            state["sums"].copy_(state["before"])
        pa.attention_weights(0, state["q"], state["lse"], state["weights"], accumulate=case["add"])
        return state["sums"]
    out, lse = torch.empty_like(state["q"]), torch.empty(state["q"].shape[:2], dtype=torch.float32, device="cuda")
    pa.decode(0, state["q"], out=out, lse=lse)
    return dict(out=out, lse=lse)


# ---- the definition in 64 bits -------------------------------------------------------------------------------


def _stands_for(x):
    """The values that x's 4-bit form stands for, group by group from the definition."""
    g = x.double().reshape(-1, GROUP)
    lo = g.min(1, keepdim=True).values
    s = ((g.max(1, keepdim=True).values - lo) / 16).to(torch.bfloat16).double()
    safe = s.masked_fill(s == 0, 1.0)
    cell = torch.div(g - lo, safe, rounding_mode="floor").clamp(0, 15)
    return torch.where(s == 0, lo.expand_as(g), lo + s * (2 * cell + 1) / 2).reshape(x.shape)


def exact(case, seed):
    x = _inputs(case, seed)
    if case["op"] == "store":
        return dict(k=_stands_for(x["k"]), v=_stands_for(x["v"]))
    st = x["st"]
    if case["op"] == "evict":
        out = []
        for k, v, w, n, four, keep in zip(x["k"], x["v"], x["w"], st["lens"], st["four"], st["keep"]):
            m = min(n, keep)
            rank = w.double().cpu().numpy().copy()
            rank[..., :case["first"]] = np.inf
            rank[..., max(0, n - case["last"]):] = np.inf
            kept = np.sort(np.argsort(-rank, axis=-1, kind="stable")[..., :m], axis=-1)
            at = torch.from_numpy(kept).cuda()
            k, v = (_stands_for(k), _stands_for(v)) if four else (k.double(), v.double())
            take = [torch.stack([torch.stack([y[layer, at[layer, h], h] for h in range(case["hkv"])], 1) for layer in range(case["layers"])]) for y in (k, v)]
            out.append(dict(kept=None, k=take[0], v=take[1], w=torch.gather(w.double(), 2, at)))
        return out
    k, v = x["k"].double(), x["v"].double()
    k[x["four"]] = _stands_for(x["k"][x["four"]])
    v[x["four"]] = _stands_for(x["v"][x["four"]])
    g, scale = case["hq"] // case["hkv"], case["d"] ** -0.5
    qd = x["q"].double().reshape(case["requests"], case["hkv"], g, case["d"])
    if case["op"] == "weights":
        lse = _attend(x["q"], _held(x["k"], x["four"]), None, x["table"])[1].double().reshape(case["requests"], case["hkv"], g)
        got = x["before"].double() if case["add"] else torch.zeros_like(x["before"], dtype=torch.float64)
        for r in range(case["requests"]):
            rows = x["table"][r][x["table"][r] >= 0]
            s = (qd[r] @ k[rows].permute(1, 2, 0)) * scale  # [hkv, g, rows]
            got[:, rows] += (s - lse[r][..., None]).exp().sum(1)
        return got
    out = torch.zeros(case["requests"], case["hkv"], g, case["d"], dtype=torch.float64, device="cuda")
    lse = torch.full((case["requests"], case["hkv"], g), -math.inf, dtype=torch.float64, device="cuda")
    for r in range(case["requests"]):
        rows = x["table"][r][x["table"][r] >= 0]
        if len(rows):
            s = (qd[r] @ k[rows].permute(1, 2, 0)) * scale
            lse[r] = torch.logsumexp(s, -1)
            out[r] = torch.softmax(s, -1) @ v[rows].transpose(0, 1)
    return dict(out=out.reshape(case["requests"], case["hq"], case["d"]), lse=lse.reshape(case["requests"], case["hq"]))
