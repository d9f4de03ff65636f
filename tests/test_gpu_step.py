"""What stands around a step's attention, against the fp64 definitions: growing nodes, projections with per-row adapters,
token log probabilities; and a whole decode loop of them."""
import math

import numpy as np
import pytest
import torch

from helpers import MAX_ABS, REL_L2, assert_close
from kv4_cases import private_workload
from oracle import attention as OA
from oracle import step as OS

pytestmark = pytest.mark.gpu


def _pa(lens=(64,), hq=8, hkv=8, d=128, layers=1, paths=None, **kw):
    from paper_2605_22566_b200.runtime import PathAttention
    return PathAttention(private_workload(list(lens), paths or [[v] for v in range(len(lens))], hq, hkv, d, layers=layers), **kw)


def _ints(*xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _bf16(rng, *shape):
    return torch.from_numpy(rng.standard_normal(shape)).to(torch.bfloat16)


# ---- nodes that grow ---------------------------------------------------------------------------------


@pytest.mark.parametrize("hkv,d,layers", [(1, 64, 1), (2, 128, 3), (3, 64, 2), (8, 128, 1)])
def test_growing_nodes_hold_what_came(hkv, d, layers):
    """Rounds of odd counts, zero among them, tokens taken back, and nodes in any order; every row and the zeros behind them."""
    rng = np.random.default_rng(hkv * d + layers)
    room = [200, 1, 64, 0, 131, 500]
    pa = _pa(room, hkv, hkv, d, layers)
    pa.pool.fill_(0xFF)                                           # NaN patterns where nothing was written
    model = OS.OpenNodes()
    for v in (2, 0, 1, 3, 5, 4):
        pa.open_node(v, room[v])
        model.open(v, room[v], pa.node_slot(v))
    for step in range(7):
        nodes = rng.permutation(6)[:rng.integers(1, 7)].tolist()
        has = [len(model.rows[v]) for v in nodes]
        held = None if step % 2 == 0 else [int(rng.integers(max(0, h - 70), h + 1)) for h in has]
        counts = [int(rng.integers(0, min(room[v] - h, 130) + 1)) for v, h in zip(nodes, held or has)]
        new = sum(counts) + 3 * (step == 3)
        wide = _bf16(rng, layers, new, (2 + 3) * hkv * d).cuda()   # K and V are parts of wider rows
        k, v = (wide[:, :, i * hkv * d:(i + 1) * hkv * d].unflatten(2, (hkv, d)) for i in (2, 4))
        slots, lens = pa.append_slots(_ints(*nodes), _ints(*counts), new, None if held is None else _ints(*held))
        for layer in range(layers):
            pa.append(layer, slots, k[layer], v[layer])
        want, want_lens = model.append(nodes, held, counts, new, [(step, i) for i in range(new)])
        assert slots.tolist() == want and lens.tolist() == want_lens
        if step == 0:
            kept = {}
        for i in range(new):
            kept[step, i] = (k[:, i].clone(), v[:, i].clone())
        for n in range(6):
            for layer in range(layers):
                got_k, got_v = pa.load_node(n, layer)              # an open node reads at its room
                ref = torch.zeros(2, room[n], hkv, d, dtype=torch.bfloat16, device="cuda")
                for t, at in enumerate(model.rows[n]):
                    ref[0, t], ref[1, t] = kept[at][0][layer], kept[at][1][layer]
                assert torch.equal(got_k.view(torch.int16), ref[0].view(torch.int16)) and torch.equal(got_v.view(torch.int16), ref[1].view(torch.int16)), (step, n)
    assert pa.status() == 0
    pa.close()


def test_slots_of_many_requests_with_refused_ones_among_them():
    from paper_2605_22566_b200 import binding as B
    rng = np.random.default_rng(3)
    n = 1500
    room = rng.integers(0, 100, n).tolist()
    pa = _pa(room, 1, 1, 64)
    model = OS.OpenNodes()
    for v in range(n):
        if v % 50 != 49:                                             # the others are not open
            pa.open_node(v, room[v])
            model.open(v, room[v], pa.node_slot(v))
    nodes = rng.permutation(n).tolist()
    counts = [int(rng.integers(-1, max(1, room[v]) + 2)) for v in nodes]  # some have no room, some are negative
    total = sum(max(c, 0) for c in counts)
    for held, new in ((None, total), ([int(rng.integers(-1, 5)) for _ in nodes], total + 40), (None, total // 2)):
        slots, lens = pa.append_slots(_ints(*nodes), _ints(*counts), new, None if held is None else _ints(*held))
        want, want_lens = model.append(nodes, held, counts, new)
        assert slots.tolist() == want and lens.tolist() == want_lens
        assert pa.status() in (B.GF_ERR_INVALID_ARG, B.GF_ERR_CAPACITY) and pa.status() == 0
    assert -1 in lens.tolist() and max(lens.tolist()) > 0
    # an id outside the nodes, and no request at all
    slots, lens = pa.append_slots(_ints(n, -1), _ints(1, 1), 2)
    assert slots.tolist() == [-1, -1] and lens.tolist() == [-1, -1] and pa.status() == B.GF_ERR_INVALID_ARG
    slots, _ = pa.append_slots(_ints(), _ints(), 3)
    assert slots.tolist() == [-1, -1, -1] and pa.status() == 0
    # only refused requests: what a step then appends goes nowhere
    before = pa.pool.clone()
    row = torch.ones(3, 1, 64, dtype=torch.bfloat16, device="cuda")
    pa.append(0, slots, row, row)
    assert torch.equal(pa.pool, before) and pa.status() == 0
    pa.append(0, _ints(1 << 30, 0x7FFFFFFF, -5), row, row)           # slots that no pool has
    assert torch.equal(pa.pool, before) and pa.status() == B.GF_ERR_INVALID_ARG
    pa.close()


@pytest.mark.parametrize("n", [297, 600, 20000])
def test_slots_of_batches_of_any_size(n):
    """More requests than multiprocessors, in blocks of one, of two and of 32; some take tokens back, whose rows are zeros in every layer."""
    rng = np.random.default_rng(n)
    few = 600
    pa = _pa([70] * few, 2, 2, 64, 3)
    model = OS.OpenNodes()
    for v in range(few):
        pa.open_node(v, 70)
        model.open(v, 70, pa.node_slot(v))
    pa.pool.fill_(0xFF)
    nodes = rng.permutation(few).tolist()[:n] + [-1] * (n - few)       # (the others are refused)
    counts = rng.integers(0, 66, n).tolist()
    for held in (None, [int(rng.integers(0, c + 1)) for c in counts]):
        new = counts if held is None else rng.integers(0, 5, n).tolist()
        before = [len(model.rows[v]) for v in range(few)]
        slots, lens = pa.append_slots(_ints(*nodes), _ints(*new), sum(new), None if held is None else _ints(*held))
        want, want_lens = model.append(nodes, held, new, sum(new))
        assert slots.tolist() == want and lens.tolist() == want_lens
    pa.status()
    for v in rng.permutation(few)[:40].tolist():
        for layer in range(3):
            k, val = pa.load_node(v, layer)
            gone = slice(len(model.rows[v]), max(before[v], len(model.rows[v])))
            assert not k[gone].any() and not val[gone].any()
    pa.close()


@pytest.mark.parametrize("n", [2, 40, 700])
def test_a_node_named_twice_in_a_batch(n):
    """The first request counts, the others are refused; near to each other and far apart."""
    from paper_2605_22566_b200 import binding as B
    rng = np.random.default_rng(n)
    pa = _pa([90] * n, 1, 1, 64)
    model = OS.OpenNodes()
    for v in range(n):
        pa.open_node(v, 90)
        model.open(v, 90, pa.node_slot(v))
    for _ in range(3):
        nodes = rng.permutation(n)
        nodes[rng.integers(0, n, n // 3 + 1)] = nodes[rng.integers(0, n, n // 3 + 1)]
        nodes[-1] = nodes[0]
        counts = rng.integers(0, 9, n).tolist()
        held = [int(rng.integers(0, len(model.rows[v]) + 1)) for v in nodes.tolist()]
        slots, lens = pa.append_slots(_ints(*nodes.tolist()), _ints(*counts), sum(counts), _ints(*held))
        want, want_lens = model.append(nodes.tolist(), held, counts, sum(counts))
        assert slots.tolist() == want and lens.tolist() == want_lens and lens.tolist()[-1] == -1
        assert pa.status() == B.GF_ERR_INVALID_ARG
    pa.close()


def test_close_reopen_release_and_refusals():
    from paper_2605_22566_b200 import binding as B
    pa = _pa([300, 64, 64, 10], 2, 2, 64, 2, extra_tiles=4, max_residual_nodes=1)
    w, hkv, d = torch.ones(300, 2, 64, dtype=torch.bfloat16, device="cuda"), 2, 64
    pa.open_node(0, 300)
    assert B.gf_node_kv_open(pa.g, 0, 300, pa.stream) == B.GF_ERR_INVALID_ARG
    assert B.gf_node_kv_open(pa.g, 1, 64 * 100, pa.stream) == B.GF_ERR_CAPACITY
    assert B.gf_node_kv_open(pa.g, 1, -1, pa.stream) == B.gf_node_kv_open(pa.g, 4, 1, pa.stream) == B.GF_ERR_INVALID_ARG
    pa.write_node(1, 0, w[:64], w[:64])
    # an open node has no length on the host
    assert B.gf_node_kv_write(pa.g, 0, 0, w.data_ptr(), w.data_ptr(), 300, pa.stream) == B.GF_ERR_INVALID_ARG
    assert B.gf_node_kv_reserve(pa.g, 0, 300, pa.stream) == B.GF_ERR_INVALID_ARG
    assert B.gf_node_kv_reconstruct(pa.g, 2, 0, 0, None, None, pa.stream) == B.GF_ERR_INVALID_ARG
    assert B.gf_node_kv_reconstruct(pa.g, 0, 0, 1, None, None, pa.stream) == B.GF_ERR_INVALID_ARG
    assert B.gf_node_kv_attach_residual(pa.g, 2, 0, 0, None, None, pa.stream) == B.GF_ERR_INVALID_ARG
    weights = pa.new_weights()
    for dst, src in ((2, 0), (0, 1)):
        with pytest.raises(B.GfError):
            pa.evict([(dst, src, 20, 1, 1)], weights)
    assert B.gf_node_kv_close(pa.g, 1, 64, pa.stream) == B.gf_node_kv_close(pa.g, 0, 301, pa.stream) == B.gf_node_kv_close(pa.g, 0, -1, pa.stream) == B.GF_ERR_INVALID_ARG
    # tables of a time before the lengths moved are stale
    pa.write_node(3, 0, w[:10], w[:10])
    pa.open_node(2, 64)
    pa.build()
    slots, _ = pa.append_slots(_ints(0), _ints(100), 100)
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.GfError):
        pa.decode(0, q)
    for layer in range(2):
        pa.append(layer, slots, w[:100] * 2, w[:100] * 3)
    used = B.gf_pool_info(pa.g).tiles_in_use
    pa.close_node(0, 70)                                             # drops the last 30 and three tiles
    assert B.gf_pool_info(pa.g).tiles_in_use == used - 3 and B.gf_node_extent(pa.g, 0)[1] == 70
    pa.build()
    assert pa.info().resident_tokens == 70 + 64 + 10
    for layer in range(2):
        k, v = pa.load_node(0, layer)
        assert bool((k == 2).all()) and bool((v == 3).all()) and k.shape[0] == 70
    # the rest of its last tile is zero: read it through a node of 128 over the same tiles
    view = pa.pool.view(torch.bfloat16).view(2, 2, -1, 2, 64, 64)
    tile = pa.node_slot(0) // 64 + 1
    assert bool((view[:, :, tile, :, 6:] == 0).all()) and bool((view[:, :, tile, 0, :6] == 2).all())
    assert pa.status() == 0
    slots, lens = pa.append_slots(_ints(0), _ints(1), 1)             # closed: no longer open
    assert slots.tolist() == [-1] and pa.status() == B.GF_ERR_INVALID_ARG
    # more than it holds is reported, the rows read as zeros
    pa.close_node(2, 5)
    assert pa.status() == B.GF_ERR_INVALID_ARG and bool((pa.load_node(2, 0)[0] == 0).all())
    assert B.gf_node_kv_release(pa.g, 0, pa.stream) == B.GF_OK and B.gf_node_kv_open(pa.g, 0, 64, pa.stream) == B.GF_OK
    assert B.gf_node_kv_release(pa.g, 0, pa.stream) == B.GF_OK       # released while open
    slots, _ = pa.append_slots(_ints(0), _ints(1), 1)
    assert slots.tolist() == [-1] and pa.status() == B.GF_ERR_INVALID_ARG
    # arguments
    for bad in (dict(layer=2), dict(layer=-1), dict(n=-1), dict(ks=65), dict(vs=-8), dict(k=8), dict(s=2), dict(v=None)):
        a = {**dict(layer=0, n=1, s=w.data_ptr(), k=w.data_ptr(), ks=128, v=w.data_ptr(), vs=128), **bad}
        if a["k"] == 8 or a["s"] == 2:
            a["k" if a["k"] == 8 else "s"] = w.data_ptr() + (8 if a["k"] == 8 else 2)
        assert B.gf_node_kv_append(pa.g, a["layer"], a["n"], a["s"], a["k"], a["ks"], a["v"], a["vs"], pa.stream) == B.GF_ERR_INVALID_ARG, bad
    p = w.data_ptr()
    for args in ((-1, p, None, p, 1, p), (1, None, None, p, 1, p), (1, p, None, None, 1, p), (1, p, None, p, 1, None), (1, p, None, p, -1, p), (1, p + 2, None, p, 1, p)):
        assert B.gf_append_slots(pa.g, *args, None, pa.stream) == B.GF_ERR_INVALID_ARG, args
    with pytest.raises(ValueError):
        pa.append(0, _ints(0), w[:1].float(), w[:1])
    with pytest.raises(ValueError):
        pa.append_slots(_ints(0, 1), _ints(1), 1)
    pa.close()


@pytest.mark.parametrize("deferred", [False, True])
def test_decode_and_extend_over_open_nodes(deferred):
    """Growing suffixes beside a shared node: each step's attention against the concatenation."""
    rng = np.random.default_rng(8)
    hq, hkv, d = 8, 2, 128
    pa = _pa([150, 200, 200, 200], hq, hkv, d, 1, [[0, 1], [0, 2], [3]])
    base = [_bf16(rng, 150, hkv, d) for _ in range(2)]
    pa.write_node(0, 0, base[0].cuda(), base[1].cuda())
    kv = {0: (base[0].double().numpy(), base[1].double().numpy())}
    for v in (1, 2, 3):
        pa.open_node(v, 200)
        kv[v] = (np.zeros((0, hkv, d)), np.zeros((0, hkv, d)))
    for counts in ([0, 1, 5], [63, 1, 100], [1, 1, 1], [64, 0, 2]):
        new = sum(counts)
        k, v = _bf16(rng, new, hkv, d), _bf16(rng, new, hkv, d)
        slots, _ = pa.append_slots(_ints(1, 2, 3), _ints(*counts), new)
        pa.build(deferred=deferred)
        pa.append(0, slots, k.cuda(), v.cuda())
        at = 0
        for i, c in enumerate(counts):
            kv[i + 1] = tuple(np.concatenate([old, x[at:at + c].double().numpy()]) for old, x in zip(kv[i + 1], (k, v)))
            at += c
        q = _bf16(rng, 3, hq, d)
        out = pa.decode(0, q.cuda())
        ref, _ = OA.decode([[0, 1], [0, 2], [3]], lambda n: kv[n], q.double().numpy(), hkv)
        assert_close(out.double().cpu().numpy(), ref, str(counts))
        assert pa.status() == 0
    if not deferred:
        from paper_2605_22566_b200 import binding as B
        pa.build(mode=B.GF_MODE_EXTEND)                            # an open node at its present length
        rows = [kv[n][0].shape[0] for n in (1, 2, 3)]
        q = _bf16(rng, sum(rows), hq, d)
        out = pa.extend(0, q.cuda())
        ref, _ = OA.extend([[0, 1], [0, 2], [3]], lambda n: kv[n], q.double().numpy(), hkv)
        assert_close(out.double().cpu().numpy(), ref, "extend")
    pa.close()


# ---- projections -------------------------------------------------------------------------------------


def _check_projection(got, x, w, a, b, scale, which):
    """A sum of n products of bf16 numbers in fp32 is off by at most n 2^-23 of the sum of their magnitudes (every addition by 2^-23 of
    what it gives, whatever the order, and truncation allowed for); the adapter's inner sums likewise, and the products with them; then one rounding
    to the output's type, half a step."""
    ref, size = OS.project(*(None if t is None else t.double().cpu().numpy() for t in (x, w, a, b, scale)), None if which is None else which.tolist())
    n = x.shape[1] + 64 + 16
    off = np.abs(got.double().cpu().numpy() - ref)
    bound = 2 * n * 2.0 ** -23 * size + np.abs(ref) * torch.finfo(got.dtype).eps / 2
    assert np.all(off <= bound * 1.001 + 1e-37), float((off / (bound + 1e-37)).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,k,n,adapters,rank", [
    (1, 8, 1, 0, 0), (1, 8, 1, 1, 8), (1, 1000, 130, 3, 16), (2, 4096, 129, 0, 0), (7, 72, 127, 2, 24), (16, 64, 128, 1, 64), (17, 2048, 500, 40, 8),
    (33, 520, 257, 5, 40), (65, 1032, 1000, 9, 16), (255, 128, 384, 3, 64), (256, 256, 256, 300, 16), (257, 320, 640, 2, 32), (600, 192, 129, 4, 48),
    (1025, 4104, 200, 7, 16), (3000, 64, 300, 17, 8), (1500, 200, 6150, 3, 64),
    (2000, 136, 5000, 1, 16), (40, 72, 40000, 6, 16), (700, 64, 20000, 0, 0)])  # (the last four: more tiles than multiprocessors)
def test_projection_sizes(rows, k, n, adapters, rank, dtype):
    from paper_2605_22566_b200.runtime import Projection
    rng = np.random.default_rng(rows * k + n)
    pa = _pa()
    x, w = _bf16(rng, rows, k).cuda(), (_bf16(rng, n, k) * k ** -0.5).cuda()
    a = b = scale = which = None
    if adapters:
        a, b = (_bf16(rng, adapters, rank, k) * k ** -0.5).cuda(), _bf16(rng, adapters, n, rank).cuda()
        scale = torch.from_numpy(rng.uniform(-1, 1, adapters)).float().cuda()
        # stretches of rows with one adapter and rows with one each
        which = np.repeat(rng.integers(-1, adapters, -(-rows // 5)), 5)[:rows]
        which[rows // 2:] = rng.integers(-1, adapters, rows - rows // 2)
        which = _ints(*which.tolist())
    p = Projection(w, a, b, scale)
    got = pa.project(p, x, which, dtype=dtype)
    _check_projection(got, x, w, a, b, scale, which)
    again = pa.project(p, x, which, dtype=dtype)
    assert torch.equal(got, again)                                   # a fixed order of additions
    if adapters:
        _check_projection(pa.project(p, x, None, dtype=dtype), x, w, None, None, None, None)   # no row has one
        assert torch.equal(pa.project(p, x, torch.full_like(which, -1), dtype=dtype), pa.project(p, x, None, dtype=dtype))
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,k,n,adapters,rank", [
    # a pair's tiles: 128, 129, 256 and 257 features, the last with two of three halves empty; K in a few and in many parts; odd numbers of stages
    (256, 192, 128, 0, 0), (256, 192, 129, 2, 16), (511, 64, 256, 3, 64), (512, 4096, 257, 0, 0), (256, 2624, 300, 3, 24), (300, 8192, 513, 5, 40),
    (2304, 72, 600, 2, 8), (2305, 128, 520, 0, 0),
    # every row its own adapter, odd numbers of slots; the ways to A x on either side of their border
    (256, 64, 300, 1000, 64), (97, 136, 200, 97, 32), (101, 64, 140, 400, 24), (592, 64, 140, 3, 32), (593, 64, 140, 3, 32), (1184, 40, 70, 9, 16), (1185, 40, 70, 9, 16),
    # tiles of 128 rows; more tiles of adapters for a tile of x than a cluster has blocks, a few more than half, and fewer
    (300, 1024, 700, 9, 24), (1294, 1400, 700, 46, 8), (1100, 1224, 40, 58, 8), (600, 2048, 300, 30, 64), (300, 4096, 140, 7, 32), (4500, 328, 60, 40, 64),
    # all the adapters that there may be; rows in more than one pass, the last of one row and of many
    (40, 16, 24, 32768, 8), (16385, 24, 40, 3, 8), (16384 + 300, 16, 33, 40, 16), (2 * 16384 + 5, 8, 16, 2, 8)])
def test_projection_at_the_borders_of_its_launches(rows, k, n, adapters, rank, dtype):
    from paper_2605_22566_b200.runtime import Projection
    rng = np.random.default_rng(rows * 3 + k + n)
    pa = _pa()
    x, w = _bf16(rng, rows, k).cuda(), (_bf16(rng, n, k) * k ** -0.5).cuda()
    a = b = scale = which = None
    if adapters:
        a, b = (_bf16(rng, adapters, rank, k) * k ** -0.5).cuda(), _bf16(rng, adapters, n, rank).cuda()
        scale = torch.from_numpy(rng.uniform(-1, 1, adapters)).float().cuda()
        which = _ints(*rng.integers(-1, adapters, rows).tolist())
        which[-1] = adapters - 1
    p = Projection(w, a, b, scale)
    got = pa.project(p, x, which, dtype=dtype)
    _check_projection(got, x, w, a, b, scale, which)
    assert torch.equal(got, pa.project(p, x, which, dtype=dtype)) and pa.status() == 0
    pa.close()


def test_projections_of_two_handles_and_threads_at_once():
    """Two threads, each with a stream of its own, with one projection; one, two and three launches a call."""
    import threading
    from paper_2605_22566_b200.runtime import Projection
    rng = np.random.default_rng(9)
    pas = [_pa(), _pa()]
    p = Projection((_bf16(rng, 900, 256) * 0.06).cuda(), (_bf16(rng, 6, 16, 256) * 0.06).cuda(), _bf16(rng, 6, 900, 16).cuda())
    xs = [_bf16(rng, rows, 256).cuda() for rows in (3, 300, 1500)]
    ids = [_ints(*rng.integers(-1, 6, len(x)).tolist()) for x in xs]
    want = [pas[0].project(p, x, i) for x, i in zip(xs, ids)]
    for y, x, i in zip(want, xs, ids):
        _check_projection(y, x, p.weight, p.a, p.b, None, i)
    torch.cuda.synchronize()
    bad = []

    def work(pa):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                got = [pa.project(p, x, i) for x, i in zip(xs, ids)]
            torch.cuda.current_stream().synchronize()
        bad.extend(n for n, (y, z) in enumerate(zip(got, want)) if not torch.equal(y, z))
    threads = [threading.Thread(target=work, args=(pa,)) for pa in pas]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
    for pa in pas:
        assert pa.status() == 0
        pa.close()


def test_projection_strides_bad_adapters_and_what_lies_beside():
    from paper_2605_22566_b200 import binding as B
    from paper_2605_22566_b200.runtime import Projection
    rng = np.random.default_rng(5)
    pa = _pa()
    wide_x, wide_w = _bf16(rng, 40, 640).cuda(), _bf16(rng, 200, 512).cuda()
    wide_x[:, 264 + 128:] = float("nan")                            # what lies behind a row is not read into a result
    wide_w[:, :64] = float("nan")
    x, w = wide_x[:, 264:264 + 128], wide_w[:, 64:192]
    a, b = _bf16(rng, 2, 8, 128).cuda(), _bf16(rng, 2, 200, 8).cuda()
    which = _ints(*([0, 1, -1, 7, -2, 1 << 30] * 7)[:40])
    whole = torch.full((42, 333), 7.0, device="cuda")
    out = whole[1:41, 20:220]
    assert pa.project(Projection(w, a, b), x, which, out=out) is out
    clean = torch.where((which >= 0) & (which < 2), which, torch.full_like(which, -1))
    _check_projection(out, x, w, a, b, None, clean)
    assert pa.status() == B.GF_ERR_INVALID_ARG and pa.status() == 0
    whole[1:41, 20:220] = 7.0
    assert bool((whole == 7.0).all())
    bf = torch.full((40, 201), 3.0, dtype=torch.bfloat16, device="cuda")
    pa.project(Projection(w, a, b), x, clean, out=bf[:, 1:])        # rows of an odd stride, not aligned
    _check_projection(bf[:, 1:], x, w, a, b, None, clean)
    assert bool((bf[:, 0] == 3.0).all())
    pa.close()


def test_projection_values_in_padding_and_infinite_rows():
    """A row with infinities or NaN spoils its own results and no other's; tiles are filled up with zeros."""
    from paper_2605_22566_b200.runtime import Projection
    rng = np.random.default_rng(6)
    pa = _pa()
    x, w = _bf16(rng, 70, 264).cuda(), _bf16(rng, 150, 264).cuda()
    a, b = _bf16(rng, 2, 16, 264).cuda(), _bf16(rng, 2, 150, 16).cuda()
    which = _ints(*[i % 3 - 1 for i in range(70)])
    p = Projection(w, a, b)
    clean = pa.project(p, x, which)
    x[5, 3], x[44, 200] = float("nan"), float("inf")
    got = pa.project(p, x, which)
    rest = [i for i in range(70) if i not in (5, 44)]
    assert torch.equal(got[rest], clean[rest]) and bool(got[5].isnan().all()) and not bool(got[44].isfinite().any())
    assert pa.project(p, x[:0], which[:0]).shape == (0, 150)
    pa.close()


@pytest.mark.parametrize("rows", [3, 200, 700])
def test_projection_captured_and_on_another_stream(rows):
    from paper_2605_22566_b200.runtime import Projection
    rng = np.random.default_rng(rows)
    pa = _pa()
    ps = [Projection((_bf16(rng, n, 512) * 0.05).cuda(), (_bf16(rng, 4, 16, 512) * 0.05).cuda(), _bf16(rng, 4, n, 16).cuda()) for n in (768, 512)]
    x = _bf16(rng, rows, 512).cuda()
    which = _ints(*rng.integers(-1, 4, rows).tolist())
    y, z = (torch.empty(rows, n, dtype=torch.bfloat16, device="cuda") for n in (768, 512))

    def chain():                                                    # the second reads what the first has just written
        pa.project(ps[0], x, which, out=y)
        pa.project(ps[1], y[:, 256:], which, out=z)
    chain()
    want = [y.clone(), z.clone()]
    side = torch.cuda.Stream()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    torch.cuda.current_stream().wait_stream(side)
    for g in graphs:
        with torch.cuda.graph(g):
            chain()
    for turn in range(4):
        if turn == 2:
            x.neg_()                                                # odd in x: the results change their sign
            want = [-t for t in want]
        y.zero_()
        z.zero_()
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(z, want[1]), turn
    # two calls at once, on two streams, each with scratch of its own
    others = [torch.empty_like(y) for _ in range(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for s, o in zip(streams, others):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                pa.project(ps[0], x, which, out=o)
        torch.cuda.synchronize()
        assert all(torch.equal(o, want[0]) for o in others)
    assert pa.status() == 0
    pa.close()


def test_projection_refusals():
    from paper_2605_22566_b200 import binding as B
    from paper_2605_22566_b200.runtime import Projection
    pa = _pa()
    w, x = torch.zeros(32, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    a, b = torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 32, 8, dtype=torch.bfloat16, device="cuda")
    y, which = torch.zeros(4, 32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    p = Projection(w, a, b)
    scratch = torch.zeros(1 << 12, device="cuda")
    good = dict(rows=4, x=x.data_ptr(), xs=64, which=which.data_ptr(), y=y.data_ptr(), ys=32, fp32=1, scratch=scratch.data_ptr(), nbytes=1 << 14)

    def call(**over):
        o = {**good, **over}
        return B.gf_adapter_project(pa.g, p.desc, o["rows"], o["x"], o["xs"], o["which"], o["y"], o["ys"], o["fp32"], o["scratch"], o["nbytes"], pa.stream)
    assert call() == B.GF_OK and call(rows=0) == B.GF_OK and call(which=None, scratch=None, nbytes=0) == B.GF_OK
    for bad in (dict(rows=-1), dict(x=None), dict(x=good["x"] + 8), dict(xs=56), dict(xs=68), dict(which=good["which"] + 2), dict(y=None), dict(y=good["y"] + 2),
                dict(ys=31), dict(fp32=2), dict(scratch=None), dict(scratch=good["scratch"] + 4)):
        assert call(**bad) == B.GF_ERR_INVALID_ARG, bad
    assert call(nbytes=B.gf_adapter_project_scratch_bytes(p.desc, 4) - 1) == B.GF_ERR_CAPACITY
    for bad in (dict(in_dim=60), dict(rank=80), dict(w_stride=60), dict(out_dim=0)):
        desc = B.ProjectionDesc(*[bad.get(n, getattr(p.desc, n)) for n, _ in p.desc._fields_])
        assert B.gf_adapter_project(pa.g, desc, 4, *[good[n] for n in ("x", "xs", "which", "y", "ys", "fp32", "scratch", "nbytes")], pa.stream) == B.GF_ERR_INVALID_ARG
    for args in ((x.float(),), (x[:, :32],), (x, which.long()), (x, which[:3]), (x, which, y[:, :31]), (x.cpu(),)):
        with pytest.raises(ValueError):
            pa.project(p, *args)
    with pytest.raises(ValueError):
        pa.project(Projection(w), x, which)
    with pytest.raises(ValueError):
        Projection(w, a)
    with pytest.raises(ValueError):
        Projection(w, a, b[:, :31].contiguous())
    for bad in (float("inf"), -float("inf"), float("nan")):
        b[1, 3, 2] = bad                                            # (it would reach rows of the other adapters)
        with pytest.raises(ValueError, match="finite"):
            Projection(w, a, b)
    desc = B.ProjectionDesc(*[B.GF_MAX_ADAPTERS + 1 if n == "num_adapters" else getattr(p.desc, n) for n, _ in p.desc._fields_])
    assert B.gf_adapter_project_scratch_bytes(desc, 4) == 0
    assert B.gf_adapter_project(pa.g, desc, 4, *[good[n] for n in ("x", "xs", "which", "y", "ys", "fp32", "scratch", "nbytes")], pa.stream) == B.GF_ERR_INVALID_ARG
    assert pa.status() == 0
    pa.close()


# ---- token log probabilities -------------------------------------------------------------------------


def _check_logprobs(got, x, tokens, top):
    """A probability's exponent d log2 e has two roundings and ex2 two units in the last place, so p is off by (|d| + 4) 2^-23 of itself; a sum is off by
    2^-23 of itself per addition, the longest chain being the entries of a thread (at least 128 share a row) and 16 joins, with one more factor
    of an exponential each; lse and the differences with it are rounded at their own size."""
    rows, v = x.shape
    host = x.double().cpu().numpy()
    chain = v / 128 + 48
    for r in range(rows):
        row = host[r].tolist()
        lp, h, lse, ids, tops = OS.token_logprobs(row, -1 if tokens is None else int(tokens[r]), top)
        assert got.top_ids[r].tolist() == ids, r
        fin = [t for t in row if math.isfinite(t)]
        d = np.abs(np.array(fin) - max(fin)) if math.isfinite(lse) else np.zeros(1)
        p = np.exp(-d) / np.exp(-d).sum()
        size = max([abs(t) for t in fin] + [1.0])
        tol = 2.0 ** -22 * (chain * 2 + float((p * (np.minimum(d, 1e3) + 4)).sum())) + 2.0 ** -23 * min(size, abs(lse) + abs(max(fin, default=0.0)) if math.isfinite(lse) else 0.0)
        spread = float((p * (np.minimum(d, 1e3) + 1) ** 2).sum()) + 4

        def near(a, b, t):
            if math.isfinite(b) and abs(b) >= 2.0 ** 128 - 2.0 ** 103:     # (half a step beyond fp32's largest: rounded, it is an infinity)
                b = math.copysign(math.inf, b)
            return (math.isnan(a) and math.isnan(b)) or a == b or abs(a - b) <= t
        assert near(float(got.lse[r]), lse, tol), (r, float(got.lse[r]), lse, tol)
        if tokens is not None:
            assert near(float(got.logprob[r]), lp, tol + 2.0 ** -23 * (abs(lp) if math.isfinite(lp) else 0)), (r, float(got.logprob[r]), lp)
        assert near(float(got.entropy[r]), h, 2.0 ** -21 * chain * spread), (r, float(got.entropy[r]), h)
        for a, b in zip(got.top_logprobs[r].tolist(), tops):
            assert near(a, b, tol + 2.0 ** -23 * (abs(b) if math.isfinite(b) else 0)), (r, a, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,v,top,stride", [(1, 1, 1, 0), (3, 2, 2, 1), (5, 7, 0, 3), (2, 33, 32, 0), (4, 127, 5, 1), (3, 1000, 32, 7), (1, 4099, 8, 0), (9, 5000, 20, 1),
                                               (1, 40001, 32, 0), (2, 70001, 17, 3), (150, 300, 3, 5), (40, 9001, 32, 2)])
def test_logprobs_sizes_and_strides(rows, v, top, stride, dtype):
    rng = np.random.default_rng(rows * v)
    pa = _pa()
    whole = torch.from_numpy(rng.standard_normal((rows, v + stride)) * 3).to(dtype).cuda()
    x = whole[:, stride // 2:stride // 2 + v]
    tokens = _ints(*rng.integers(0, v, rows).tolist())
    got = pa.token_logprobs(x, tokens, top)
    _check_logprobs(got, x, tokens, top)
    assert all(torch.equal(a, b) for a, b in zip(got, pa.token_logprobs(x, tokens, top)))
    if top:
        none = pa.token_logprobs(x, None, 0)
        assert none.logprob is None and torch.equal(none.lse, got.lse) and torch.equal(none.entropy, got.entropy)
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,v,top", [(1, 1000003, 32), (149, 12000, 5), (148, 12001, 5), (2100, 257, 1), (37, 30011, 2)])
def test_logprobs_of_long_and_of_many_rows(rows, v, top, dtype):
    """Rows in one part and in several, with values on a coarse grid, so that many are equal."""
    rng = np.random.default_rng(rows + v)
    pa = _pa()
    x = torch.from_numpy(np.round(rng.standard_normal((rows, v)) * 8) / 4).to(dtype).cuda()
    tokens = _ints(*rng.integers(-1, v, rows).tolist())
    _check_logprobs(pa.token_logprobs(x, tokens, top), x, tokens, top)
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("v", [40, 3001, 70001])
def test_logprobs_values_where_they_can_go_wrong(v, dtype):
    """Masked rows, ties, sorted rows, one certain token, far apart and lowest values, infinities, NaN, zeros of both signs; tokens that do not exist."""
    rng = np.random.default_rng(v)
    low = torch.finfo(dtype).min
    x = torch.from_numpy(rng.standard_normal((20, v)) * 2).to(dtype)
    x[0] = -math.inf
    x[1] = -math.inf
    x[1, v - 1] = 3.0
    x[2, rng.random(v) < 0.95] = -math.inf
    x[3] = 0.5                                                       # all equal
    x[4] = torch.from_numpy(np.sort(x[4].double().numpy())).to(dtype)       # every entry is the largest so far
    x[5] = torch.from_numpy(np.sort(x[5].double().numpy())[::-1].copy()).to(dtype)
    x[6, v // 2] = 90.0                                              # nearly certain
    x[7] = x[7] * 40
    x[8] = low
    x[9] = low
    x[9, 5] = 1.0
    x[10, 7] = math.nan
    x[11, 8] = math.inf
    x[12] = math.nan
    x[13] = 0.0
    x[13, ::2] = -0.0
    x[14] = torch.from_numpy(np.where(np.arange(v) % 3 == 0, 1.5, -2.0)).to(dtype)   # many at the top
    x[15, :] = x[15, :] + 300
    x[16, :] = x[16, :] - 300
    x[17, : v // 2] = -math.inf
    x[18, v // 2:] = math.nan
    x[19] = -math.inf
    x[19, 3] = math.nan
    x = x.cuda()
    tokens = _ints(*([0, v - 1, 1, v - 1, v, 2, v // 2, -1, 3, 5, 7, 8, 0, 1, -2, 0, 0, 0, 0x7FFFFFFF, 3][:20]))
    pa = _pa()
    top = min(32, v)
    got = pa.token_logprobs(x, tokens, top)
    _check_logprobs(got, x, tokens, top)
    assert all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(got, pa.token_logprobs(x, tokens, top)))
    pa.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("v", [9, 300, 20003])
def test_logprobs_where_differences_pass_the_range_of_fp32(v, dtype):
    """Largest logits on either side of 1e38, the others at the ends of the range, with masked ones among them."""
    rng = np.random.default_rng(v)
    pa = _pa()
    ends = np.array([-3.38e38, -1.3e38, -1.21e38, -1.19e38, -1e38, -math.inf])
    tops = [-1.01e38, -9.9e37, -9e37, 0.0, 9e37, 9.9e37, 1.01e38, 3.38e38]
    x = rng.choice(ends, (len(tops), v))
    for r, top in enumerate(tops):
        x[r] = np.minimum(x[r], top)
        x[r, rng.integers(0, v, 3)] = top
    x = torch.from_numpy(x).to(dtype).cuda()
    tokens = _ints(*rng.integers(0, v, len(tops)).tolist())
    _check_logprobs(pa.token_logprobs(x, tokens, 7), x, tokens, 7)
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("v", [61, 2500, 40009])
def test_logprobs_of_large_logits_and_finite_masks(v, dtype):
    """Logits far from zero and close to each other, on either side of where differences are formed in another way; rows of which a finite mask
    leaves a few entries, one, or none."""
    rng = np.random.default_rng(v)
    pa = _pa()
    rows = [base + rng.standard_normal(v) * 3 for base in (-3e6, -1e6, -1e3, 4e3, 9.99995e5, 1e6, 1.00001e6, 5e7, 2e12)]
    for mask in (-1e4, -65504.0, -1e9, -1e30, float(torch.finfo(dtype).min)):
        for left in (v // 20, 3, 1, 0):
            row = np.full(v, mask)
            row[rng.permutation(v)[:left]] = rng.standard_normal(left) * 3
            rows.append(row)
    x = torch.from_numpy(np.stack(rows)).to(dtype).cuda()
    tokens = _ints(*x.argmax(1).tolist())
    _check_logprobs(pa.token_logprobs(x, tokens, 5), x, tokens, 5)
    assert pa.status() == 0
    pa.close()


def test_logprobs_of_many_rows_captured_and_refusals():
    from paper_2605_22566_b200 import binding as B
    rng = np.random.default_rng(4)
    pa = _pa()
    x = torch.from_numpy(rng.standard_normal((700, 1501)) * 2).to(torch.bfloat16).cuda()
    tokens = _ints(*rng.integers(-1, 1501, 700).tolist())
    want = pa.token_logprobs(x, tokens, 4)
    _check_logprobs(want, x, tokens, 4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = pa.token_logprobs(x, tokens, 4)
    for _ in range(2):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert pa.token_logprobs(x[:0], tokens[:0], 2).top_ids.shape == (0, 2)
    f = torch.zeros(4, 16, device="cuda")
    p, i = f.data_ptr(), tokens.data_ptr()
    good = dict(rows=4, v=16, x=p, s=16, fp32=1, t=i, top=2, lp=p, ids=i)

    def call(**over):
        o = {**good, **over}
        return B.gf_token_logprobs(pa.g, o["rows"], o["v"], o["x"], o["s"], o["fp32"], o["t"], o["top"], B.Logprobs(o["lp"], None, None, o["ids"], None), pa.stream)
    scratch_ids, scratch_lp = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    good.update(ids=scratch_ids.data_ptr(), lp=scratch_lp.data_ptr())
    assert call() == B.GF_OK and call(rows=0, x=None) == B.GF_OK and call(ids=None, lp=None, t=None) == B.GF_OK
    for bad in (dict(rows=-1), dict(v=0), dict(x=None), dict(x=p + 2), dict(s=15), dict(fp32=2), dict(t=None), dict(t=i + 1), dict(top=33), dict(top=-1), dict(v=1, s=1),
                dict(lp=good["lp"] + 2), dict(ids=good["ids"] + 2)):
        assert call(**bad) == B.GF_ERR_INVALID_ARG, bad
    for args in ((x.half(),), (x.t(),), (x, tokens.long()), (x, tokens[:3]), (x, tokens, 33), (x[:, :3], tokens, 4), (x.cpu(),)):
        with pytest.raises(ValueError):
            pa.token_logprobs(*args)
    assert pa.status() == 0
    pa.close()


# ---- a decode loop -----------------------------------------------------------------------------------


@pytest.mark.parametrize("captured", [False, True])
def test_a_decode_loop(captured):
    """Hidden rows -> queries, keys and values under each request's adapter -> appended -> tables -> attention over the paths -> output projection
    -> logits -> the next tokens, several steps in a row, against the same in fp64 from the bf16 values that each stage was given."""
    from paper_2605_22566_b200.runtime import Projection
    rng = np.random.default_rng(12)
    hq, hkv, d, hidden, vocab, requests = 8, 2, 64, 256, 500, 5
    paths = [[0, 2 + r] if r % 2 else [1, 2 + r] for r in range(requests)]
    pa = _pa([90, 33] + [70] * requests, hq, hkv, d, 1, paths)
    kv = {}
    for v, n in ((0, 90), (1, 33)):
        k, val = _bf16(rng, n, hkv, d), _bf16(rng, n, hkv, d)
        pa.write_node(v, 0, k.cuda(), val.cuda())
        kv[v] = [k.double().numpy(), val.double().numpy()]
    for r in range(requests):
        pa.open_node(2 + r, 70)
        kv[2 + r] = [np.zeros((0, hkv, d)), np.zeros((0, hkv, d))]
    width = (hq + 2 * hkv) * d
    mk = lambda n, k: Projection((_bf16(rng, n, k) * k ** -0.5).cuda(), (_bf16(rng, 3, 16, k) * k ** -0.5).cuda(), (_bf16(rng, 3, n, 16) * 0.3).cuda())  # noqa: E731
    qkv_p, out_p, head = mk(width, hidden), mk(hidden, hq * d), Projection((_bf16(rng, vocab, hidden) * 0.2).cuda())
    embed = _bf16(rng, vocab, hidden).cuda()
    which, nodes, one = _ints(*[r % 4 - 1 for r in range(requests)]), _ints(*range(2, 2 + requests)), torch.ones(requests, dtype=torch.int32, device="cuda")
    tokens = _ints(*rng.integers(0, vocab, requests).tolist())
    pa.build(deferred=True)
    state = {}

    def step():
        x = embed[tokens.long()]
        qkv = pa.project(qkv_p, x, which)
        slots, lens = pa.append_slots(nodes, one, requests)
        pa.build(deferred=True)
        pa.append(0, slots, qkv[:, hq * d:(hq + hkv) * d].view(requests, hkv, d), qkv[:, (hq + hkv) * d:].view(requests, hkv, d))
        q = qkv[:, :hq * d].contiguous().view(requests, hq, d)
        out = torch.empty_like(q)
        pa.decode(0, q, out=out)
        y = pa.project(out_p, out.view(requests, hq * d), which)
        logits = pa.project(head, y, dtype=torch.float32)
        got = pa.token_logprobs(logits, None, 3)
        state.update(x=x, qkv=qkv, out=out, y=y, logits=logits, got=got, lens=lens, given=tokens.clone())
        tokens.copy_(got.top_ids[:, 0])
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    for n in range(1, 9):
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        s = state
        assert s["lens"].tolist() == [n] * requests
        _check_projection(s["qkv"], s["x"], qkv_p.weight, qkv_p.a, qkv_p.b, None, which)
        rows = s["qkv"].double().cpu().numpy()
        for r in range(requests):
            for i in (0, 1):
                new = rows[r, (hq + i * hkv) * d:(hq + (i + 1) * hkv) * d].reshape(1, hkv, d)
                kv[2 + r][i] = np.concatenate([kv[2 + r][i], new])
        ref, _ = OA.decode(paths, lambda v: kv[v], rows[:, :hq * d].reshape(requests, hq, d), hkv)
        # (values of a few tokens reach beyond 4, where half a step of bf16, 2^-8 of the value, is more than the tolerance for values near 1)
        off = np.abs(s["out"].double().cpu().numpy() - ref)
        assert np.all(off <= MAX_ABS + 2.0 ** -8 * np.abs(ref)) and np.linalg.norm(off) <= REL_L2 * np.linalg.norm(ref), n
        _check_projection(s["y"], s["out"].view(requests, -1), out_p.weight, out_p.a, out_p.b, None, which)
        _check_projection(s["logits"], s["y"], head.weight, None, None, None, None)
        _check_logprobs(s["got"], s["logits"], None, 3)
        assert tokens.tolist() == s["got"].top_ids[:, 0].tolist()
    assert pa.status() == 0
    if captured:
        del graph
    pa.close()
