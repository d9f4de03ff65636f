"""Timed cases of what stands on both sides of a decode step's attention.

  append    the token slots of a batch's new tokens, worked out from the requests' lengths, and their K/V rows put into the
            growing nodes (gf_append_slots, gf_node_kv_append)
  project   a projection that all requests share with the low-rank adapters that each has of its own (gf_adapter_project)
  logprobs  log probabilities of given tokens, entropy and the top alternatives of a batch of logits (gf_token_logprobs)

The pool holds 64 tokens of one KV head per tile: K, then V, each as head_dim / 64 blocks of [64 tokens][8 chunks of 8 entries],
the chunk c of token row t at place c xor (t mod 8).

Values follow the seed; lengths, counts and which adapter a row has follow the case (its "layout")."""
import math
import random

import numpy as np
import torch

own = False

TILE = 64


def listed():
    """What each stands for: one request's next token (latency alone); a batch's next tokens; prompts that come in chunks of any length.  One token's
    query, key and value projection; the same for a batch under 64 adapters; odd sizes with fp32 outputs; a batch of prompts; a vocabulary's
    logits in fp32.  One row of logits; rows of an odd length in fp32 with many alternatives; a batch whose grammar masks most of
    the vocabulary; the scoring of long answers."""
    return [
        dict(name="append-1", op="append", requests=1, hkv=4, d=64, most=1, held=100, layout=1),
        dict(name="append-256", op="append", requests=256, hkv=8, d=128, most=1, held=300, layout=2),
        dict(name="append-chunks", op="append", requests=64, hkv=8, d=128, most=600, held=300, layout=3),
        dict(name="project-1", op="project", rows=1, k=4096, n=6144, adapters=16, rank=16, runs=1, fp32=False, layout=4),
        dict(name="project-256", op="project", rows=256, k=4096, n=6144, adapters=64, rank=16, runs=256, fp32=False, layout=5),
        dict(name="project-odd", op="project", rows=77, k=1000, n=999, adapters=5, rank=8, runs=30, fp32=True, layout=6),
        dict(name="project-prompts", op="project", rows=8192, k=4096, n=6144, adapters=12, rank=64, runs=20, fp32=False, layout=7),
        dict(name="project-logits", op="project", rows=64, k=4096, n=128000, adapters=0, rank=0, runs=64, fp32=True, layout=8),
        dict(name="logprobs-1", op="logprobs", rows=1, v=128000, fp32=False, top=8, masked=0.0, layout=9),
        dict(name="logprobs-odd", op="logprobs", rows=33, v=50001, fp32=True, top=20, masked=0.0, layout=10),
        dict(name="logprobs-masked", op="logprobs", rows=256, v=128000, fp32=False, top=5, masked=0.95, layout=11),
        dict(name="logprobs-2048", op="logprobs", rows=2048, v=128000, fp32=False, top=1, masked=0.0, layout=12),
    ]


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithms."""
    def between(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    op = rng.choice(["append", "project", "project", "logprobs"])
    layout = rng.randrange(1 << 20)
    if op == "append":
        hkv, d = rng.choice([(8, 128), (4, 64), (2, 128), (4, 128)])
        requests = between(1, 512)
        return dict(op=op, requests=requests, hkv=hkv, d=d, most=between(1, max(2, min(600, 16000 // requests))), held=between(1, 300), layout=layout)
    if op == "project":
        rows = between(1, 8192)
        return dict(op=op, rows=rows, k=8 * between(8, 768), n=between(17, 6144), adapters=between(1, 64), rank=rng.choice([8, 16, 32, 64]),
                    runs=rows if rng.random() < 0.5 else between(1, rows), fp32=rng.choice([True, False]), layout=layout)
    return dict(op=op, rows=between(1, 1024), v=between(40, 128000), fp32=rng.choice([True, False]), top=rng.choice([0, 1, 5, 20, 32]),
                masked=rng.choice([0.0, 0.0, 0.95]), layout=layout)


# ---- what a case consists of (from the case alone) ---------------------------------------------------------


def _batch(case):
    """An append batch: tokens held and tokens that come per request, the node of each (in an order of their own) and its first
    tile.  One request in eight has nothing new where prompts come in chunks."""
    rng = random.Random(case["layout"])
    n = case["requests"]
    held = [rng.randint(0, case["held"]) for _ in range(n)]
    count = [1 if case["most"] == 1 else 0 if i % 8 == 7 else rng.randint(1, case["most"]) for i in range(n)]
    node = list(range(n))
    rng.shuffle(node)
    room = [0] * n
    for h, c, v in zip(held, count, node):
        room[v] = h + c + rng.randint(0, 64)
    tiles = [-(-r // TILE) for r in room]
    first = np.concatenate([[0], np.cumsum(tiles)])
    return dict(held=held, count=count, node=node, room=room, first=[int(first[v]) for v in node], tiles=max(1, int(first[-1])), new=sum(count))


def _adapters(case):
    """Every row's adapter: `runs` stretches of neighbouring rows share one; about one stretch in six has none (-1)."""
    rng = random.Random(case["layout"])
    cuts = sorted(rng.sample(range(1, case["rows"]), case["runs"] - 1)) if case["runs"] > 1 else []
    out = []
    for a, b in zip([0] + cuts, cuts + [case["rows"]]):
        out += [-1 if not case["adapters"] or (rng.random() < 0.17 and case["rows"] > 1) else rng.randrange(case["adapters"])] * (b - a)
    return out


def work(case):
    """Bytes that no implementation can do without, every input once and every output once, and the products' operations."""
    if case["op"] == "append":
        t = _batch(case)["new"]
        return dict(bytes=8 * t * case["hkv"] * case["d"] + 4 * t + 16 * case["requests"], flops=2 * t)
    if case["op"] == "logprobs":
        r, v = case["rows"], case["v"]
        return dict(bytes=r * v * (4 if case["fp32"] else 2) + r * (16 + 8 * case["top"]), flops=4 * r * v)
    t, k, n, which = case["rows"], case["k"], case["n"], _adapters(case)
    used, with_one = len(set(which) - {-1}), sum(a >= 0 for a in which)
    return dict(bytes=2 * n * k + 2 * t * k + (4 if case["fp32"] else 2) * t * n + 2 * used * case["rank"] * (k + n) + 4 * t,
                flops=2 * t * n * k + 2 * with_one * case["rank"] * (k + n))


# ---- inputs --------------------------------------------------------------------------------------------


def _inputs(case, seed):
    """The tensors of a case, from the seed."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")
    if case["op"] == "append":
        b = _batch(case)
        hkv, d = case["hkv"], case["d"]
        # keys and values come out of one projection, beside the queries
        qkv = randn(b["new"], (4 + 2) * hkv * d).to(torch.bfloat16)
        k, v = (qkv[:, i * hkv * d:(i + 1) * hkv * d].view(b["new"], hkv, d) for i in (4, 5))
        before = randn(2, sum(b["held"]), hkv, d).to(torch.bfloat16)
        ints = {name: torch.tensor(b[name], dtype=torch.int32, device="cuda") for name in ("held", "count", "node", "first")}
        return dict(b=b, k=k, v=v, before=before, **ints)
    if case["op"] == "project":
        k, n, r, a = case["k"], case["n"], case["rank"], case["adapters"]
        out = dict(x=randn(case["rows"], k).to(torch.bfloat16), w=(randn(n, k) * k ** -0.5).to(torch.bfloat16))
        if a:
            out.update(a=(randn(a, r, k) * k ** -0.5).to(torch.bfloat16), b=(randn(a, n, r) * 0.5).to(torch.bfloat16),
                       scale=torch.rand(a, generator=gen, device="cuda") * 2 / r ** 0.5)
            out["which"] = torch.tensor(_adapters(case), dtype=torch.int32, device="cuda")
        return out
    r, v = case["rows"], case["v"]
    x = randn(r, v) * 2.5
    # a few tokens stand out, by how much differs from row to row
    bumps = torch.randint(0, v, (r, 8), generator=gen, device="cuda")
    x.scatter_add_(1, bumps, randn(r, 8).abs() * 6 * torch.rand(r, 1, generator=gen, device="cuda") + 1)
    tokens = torch.where(torch.rand(r, generator=gen, device="cuda") < 0.7, bumps[:, 0], torch.randint(0, v, (r,), generator=gen, device="cuda"))
    tokens[5::16] = -1  # rows with no token to score
    if case["masked"]:
        x.masked_fill_(torch.rand(r, v, generator=gen, device="cuda") < case["masked"], -math.inf)
        x[7::32] = -math.inf  # rows whose mask leaves nothing
    return dict(x=x.to(torch.float32 if case["fp32"] else torch.bfloat16), tokens=tokens.to(torch.int32))


def prepare(case, seed):
    x = _inputs(case, seed)
    state = dict(case=case, **x)
    if case["op"] == "append":
        b, start = x["b"], torch.tensor(x["b"]["held"], dtype=torch.int32, device="cuda")
        if own:
            pa = _handle(b["room"], case["hkv"], case["d"])
            pa.pool.zero_()
            for node, room in enumerate(b["room"]):
                pa.open_node(node, room)
            slots, _ = pa.append_slots(x["node"], start, sum(b["held"]))
            pa.append(0, slots, x["before"][0], x["before"][1])
            torch.cuda.synchronize()
            state["pa"], state["pool"] = pa, pa.pool.view(torch.bfloat16).view(case["hkv"], b["tiles"], 2, case["d"] // 64, TILE, 8, 8)
        else:
            state["pool"] = torch.zeros(case["hkv"], b["tiles"], 2, case["d"] // 64, TILE, 8, 8, dtype=torch.bfloat16, device="cuda")
            _put(state["pool"], _slots(x["first"], torch.zeros_like(start), start, sum(b["held"])), x["before"][0], x["before"][1])
    elif own:
        from paper_2605_22566_b200 import runtime
        state["pa"] = _handle([1], 8, 128)
        if case["op"] == "project":
            state["projection"] = runtime.Projection(x["w"], x.get("a"), x.get("b"), x.get("scale"))
    return state


def _handle(room, hkv, d):
    """A wGraph handle with a private node for every request, its pool sized to fit."""
    from paper_2605_22566_b200 import runtime, workloads
    n = len(room)
    w = workloads.Workload(name="operators", config_id=-1, seed=0, mode="decode", num_layers=1, num_q_heads=4 * hkv, num_kv_heads=hkv, head_dim=d,
                           num_shared_nodes=0, num_nodes=n, edge_src=np.zeros(0, np.int32), edge_dst=np.zeros(0, np.int32),
                           node_len=np.array(room, np.int32), path_ptr=np.arange(n + 1, dtype=np.int32), path_node=np.arange(n, dtype=np.int32))
    return runtime.PathAttention(w)


# ---- the operators' plain forms --------------------------------------------------------------------------


def _slots(first, held, count, new):
    """The token slot of every new row."""
    request = torch.repeat_interleave(torch.arange(len(count), device=count.device), count.long(), output_size=new)
    begin = torch.cumsum(count, 0) - count
    return (first[request] * TILE + held[request] + torch.arange(new, device=count.device) - begin[request]).int()


def _put(pool, slots, k, v):
    """The rows k, v [new, hkv, d] into the pool's places of their slots."""
    new, hkv, d = k.shape
    tile, row = (slots // TILE).view(-1, 1, 1, 1).long(), (slots % TILE).view(-1, 1, 1, 1).long()
    head = torch.arange(hkv, device=k.device).view(1, -1, 1, 1)
    block = torch.arange(d // 64, device=k.device).view(1, 1, -1, 1)
    place = torch.arange(8, device=k.device) ^ (row % 8)
    pool[head, tile, 0, block, row, place] = k.reshape(new, hkv, d // 64, 8, 8)
    pool[head, tile, 1, block, row, place] = v.reshape(new, hkv, d // 64, 8, 8)


def _project(x, w, a, b, scale, which, kind):
    """x W^T and, through all adapters with the others' parts of every row set to zero, the rows' own; in 32 bits, rounded at the end."""
    y = x.float() @ w.float().t()
    if a is not None:
        n, r, k = a.shape
        h = (x.float() @ a.float().reshape(n * r, k).t()).view(-1, n, r)
        mine = (which.view(-1, 1) == torch.arange(n, device=x.device)).float() * scale
        y = y + (h * mine.unsqueeze(-1)).flatten(1) @ b.float().transpose(1, 2).reshape(n * r, -1)
    return y.to(kind)


def _logprobs(x, tokens, top):
    """All in 32 bits.  A row with no probability anywhere has lse and every log probability at minus infinity, and no entropy."""
    x = x.float()
    m = x.amax(-1, keepdim=True).clamp(min=-3e38)
    lse = m + torch.log(torch.exp(x - m).sum(-1, keepdim=True))
    logp = torch.where(lse == -math.inf, lse, x - lse)
    p = torch.exp(logp)
    entropy = torch.where(p > 0, -p * logp, torch.zeros_like(p)).sum(-1)
    given = torch.gather(logp, 1, tokens.clamp(min=0).long().unsqueeze(1)).squeeze(1)
    out = dict(logprob=torch.where(tokens == -1, torch.zeros_like(given), given), entropy=entropy, lse=lse.squeeze(1))
    if top:
        ids = torch.sort(x, dim=-1, descending=True, stable=True)[1][:, :top]  # ties to the lowest id
        out.update(top_ids=ids.int(), top_logprobs=torch.gather(logp, 1, ids))
    return out


def run(state):
    case = state["case"]
    if own:
        return _run_own(state)
    if case["op"] == "append":
        slots = _slots(state["first"], state["held"], state["count"], state["b"]["new"])
        _put(state["pool"], slots, state["k"], state["v"])
        return dict(slots=slots, lens=state["held"] + state["count"], pool=state["pool"])
    if case["op"] == "project":
        return _project(state["x"], state["w"], state.get("a"), state.get("b"), state.get("scale"), state.get("which"),
                        torch.float32 if case["fp32"] else torch.bfloat16)
    return _logprobs(state["x"], state["tokens"], case["top"])


def _run_own(state):
    case, pa = state["case"], state["pa"]
    if case["op"] == "append":
        slots, lens = pa.append_slots(state["node"], state["count"], state["b"]["new"], held=state["held"])
        pa.append(0, slots, state["k"], state["v"])
        return dict(slots=slots, lens=lens, pool=state["pool"])
    if case["op"] == "project":
        return pa.project(state["projection"], state["x"], state.get("which"), dtype=torch.float32 if case["fp32"] else torch.bfloat16)
    got = pa.token_logprobs(state["x"], state["tokens"], case["top"])
    out = dict(logprob=got.logprob, entropy=got.entropy, lse=got.lse)
    if case["top"]:
        out.update(top_ids=got.top_ids, top_logprobs=got.top_logprobs)
    return out


# ---- the definition in 64 bits -------------------------------------------------------------------------------


def exact(case, seed):
    x = _inputs(case, seed)
    if case["op"] == "append":
        b, hkv, d = x["b"], case["hkv"], case["d"]
        pool = np.zeros((hkv, b["tiles"], 2, d // 64, TILE, 8, 8))
        rows = [[y.double().cpu().numpy() for y in (x["before"][i], z)] for i, z in enumerate((x["k"], x["v"]))]
        at = [0, 0]
        for held, count, first in zip(b["held"], b["count"], b["first"]):
            for j, (begin, n) in enumerate(((0, held), (held, count))):
                for t in range(n):
                    tile, row = first + (begin + t) // TILE, (begin + t) % TILE
                    for i in (0, 1):
                        y = rows[i][j][at[j]].reshape(hkv, d // 64, 8, 8)
                        pool[:, tile, i, :, row] = y[:, :, [c ^ (row % 8) for c in range(8)]]  # (its own inverse)
                    at[j] += 1
        return dict(slots=None, lens=None, pool=torch.from_numpy(pool).cuda())
    if case["op"] == "project":
        y = x["x"].double() @ x["w"].double().T
        if "a" in x:
            for i in range(case["adapters"]):
                rows = x["which"] == i
                y[rows] += x["scale"][i].double() * (x["x"][rows].double() @ x["a"][i].double().T @ x["b"][i].double().T)
        return y
    # a few rows at a time
    got = {name: [] for name in ("logprob", "entropy", "lse", "top_logprobs")}
    for i in range(0, case["rows"], 64):
        y, token = x["x"][i:i + 64].double(), x["tokens"][i:i + 64].long()
        empty = (y == -math.inf).all(1)
        lse = torch.logsumexp(y, 1)
        p = torch.softmax(y, 1).masked_fill(empty[:, None], 0.0)
        got["lse"].append(lse)
        got["entropy"].append((p * (lse[:, None] - y)).masked_fill(p == 0, 0.0).sum(1))
        given = (y[torch.arange(len(y)), token.clamp(min=0)] - lse).masked_fill(empty, -math.inf)
        got["logprob"].append(given.masked_fill(token == -1, 0.0))
        if case["top"]:
            got["top_logprobs"].append((torch.topk(y, case["top"], dim=1).values - lse[:, None]).masked_fill(empty[:, None], -math.inf))
    out = {name: torch.cat(v) if v else None for name, v in got.items()}
    if case["top"]:
        out["top_ids"] = None
    else:
        del out["top_logprobs"]
    return out
