"""What stands around a step's attention, at the edges of its contract: refused requests, rows that are not there, entries that are no numbers,
the digits that results hold."""
import numpy as np
import pytest
import torch

import step_digits as D
from helpers import assert_close
from kv4_cases import private_workload
from oracle import attention as OA
from oracle import eviction as OE
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


@pytest.mark.parametrize("many", [1, 3, 700])
def test_refused_requests_leave_every_row_as_it_was(many):
    """Negative and huge counts and lengths, nodes that are not open or do not exist: no entry of the pool changes, in any layer, and the nodes
    hold what they held.  Requests one to a block and many to a block; accepted ones among them take back only their own."""
    from paper_2605_22566_b200 import binding as B
    rng = np.random.default_rng(many)
    least, most = -2 ** 31, 2 ** 31 - 1
    pa = _pa([100, 100, 70, 64] + [10] * many, 2, 2, 64, 3)
    model = OS.OpenNodes()
    for v in [0, 1, 2] + list(range(4, 4 + many)):
        pa.open_node(v, 64 if v < 4 else 10)
        model.open(v, 64 if v < 4 else 10, pa.node_slot(v))
    pa.write_node(3, 0, *[_bf16(rng, 64, 2, 64).cuda()] * 2)             # written, not open
    pa.append_slots(_ints(0, 2), _ints(40, 7), 47)
    model.append([0, 2], None, [40, 7], 47)
    pa.pool.copy_(torch.from_numpy(rng.integers(0, 256, pa.pool.numel(), dtype=np.uint8)))
    before = pa.pool.clone()
    bad = [(0, 40, -1), (0, 40, least), (0, -1, 0), (0, least, 5), (0, 41, 0), (0, most, 1), (0, 3, most), (1, -1, -1), (1, 0, -1), (1, 1, 1), (1, 0, 65),
           (2, most, most), (3, 0, 1), (3, 60, 0), (3, -1, -1), (-1, -1, -1), (-1, 0, 3), (4 + many, -5, -5), (most, 0, -1), (least, least, least)]
    assert pa.status() == 0
    for node, held, count in bad:
        nodes, helds, counts = [node] + [-1] * (many - 1), [held] * many, [count] * many
        slots, lens = pa.append_slots(_ints(*nodes), _ints(*counts), 2, _ints(*helds))
        assert slots.tolist() == [-1, -1] and lens.tolist() == [-1] * many, (node, held, count)
        assert pa.status() in (B.GF_ERR_INVALID_ARG, B.GF_ERR_CAPACITY) and torch.equal(pa.pool, before), (node, held, count)
    slots, lens = pa.append_slots(_ints(*[0] * many), _ints(*[-1] * many), 0)     # held: all that it holds
    assert lens.tolist() == [-1] * many and pa.status() == B.GF_ERR_INVALID_ARG and torch.equal(pa.pool, before)
    # one request that takes tokens back between refused ones: its rows from 5 to 40 become zeros, no others do
    nodes, held, counts = [1] + [0] + [2], [-1, 5, 8], [-1, 0, 0]
    slots, lens = pa.append_slots(_ints(*nodes), _ints(*counts), 1, _ints(*held))
    assert (slots.tolist(), lens.tolist()) == model.append(nodes, held, counts, 1) and lens.tolist() == [-1, 5, -1]
    assert pa.status() == B.GF_ERR_INVALID_ARG
    view, old = (p.view(torch.int16).view(3, 2, -1, 2, 64, 64) for p in (pa.pool, before))      # [layer, head, tile, K or V, token, entries]
    at = pa.node_slot(0)
    want = old.clone()
    want[:, :, at // 64, :, 5:40] = 0
    assert torch.equal(view, want)
    pa.close()


# ---- waits that ran out --------------------------------------------------------------------------------


def test_calls_behind_a_wait_that_ran_out_end_and_the_next_ones_are_right():
    """A wait that gave up makes the waits behind it give up too, copies and all: those calls end, the report says so once, and the next calls give
    what they gave before."""
    from paper_2605_22566_b200 import binding as B
    from paper_2605_22566_b200.runtime import Projection
    rng = np.random.default_rng(1)
    pa = _pa()
    logits = [torch.from_numpy(rng.standard_normal((rows, v)) * 3).to(kind).cuda() for rows, v, kind in ((1, 40000, torch.bfloat16), (400, 9000, torch.float32))]
    p = Projection((_bf16(rng, 900, 512) * 0.05).cuda(), (_bf16(rng, 6, 16, 512) * 0.05).cuda(), _bf16(rng, 6, 900, 16).cuda())
    xs = [_bf16(rng, rows, 512).cuda() for rows in (3, 300, 1500)]
    ids = [_ints(*rng.integers(-1, 6, len(x)).tolist()) for x in xs]

    def calls():
        return [t for x in logits for t in pa.token_logprobs(x, None, 9)[1:]] + [pa.project(p, x, i, dtype=d) for x, i in zip(xs, ids) for d in (torch.bfloat16, torch.float32)]
    want = calls()
    assert pa.status() == 0
    for _ in range(3):
        st, gave_up = B.gf_debug_wait_probe(pa.g, 5000, pa.stream)
        assert st == B.GF_OK and gave_up == 1
        calls()
        assert pa.status() == B.GF_ERR_TIMEOUT and pa.status() == 0
        assert all(torch.equal(a, b) for a, b in zip(calls(), want)) and pa.status() == 0
    pa.close()


# ---- digits of projections -----------------------------------------------------------------------------


@pytest.mark.parametrize("rows,k,n", [
    # K in parts and whole, tiles of one block of 16 to 128 rows and of two with 256; 128 features and fewer
    (5, 16384, 129), (100, 16384, 700), (100, 8192, 20000), (255, 16384, 520), (256, 16384, 300), (2048, 8192, 2500), (300, 16384, 100), (700, 8200, 40)])
def test_fp32_results_hold_their_digits_over_long_sums(rows, k, n):
    """All products of one sign: additions that are cut off all take away, and what is not taken out in time shows in the norm."""
    from paper_2605_22566_b200.runtime import Projection
    pa = _pa()
    x, w = (t.cuda() for t in D.same_sign(rows, k, n, k))
    got = pa.project(Projection(w), x, dtype=torch.float32).double()
    ref = x.double() @ w.double().T
    off = float((got - ref).norm() / ref.norm())
    assert off <= D.SAME_SIGN + 2.0 ** -24, off                         # (and the result's rounding)
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,n,rank", [(1, 200, 8), (3, 300, 16), (100, 300, 24), (100, 129, 64), (255, 260, 32), (300, 600, 16), (700, 130, 64), (2000, 100, 32), (2300, 700, 8)])
def test_adapters_hold_their_digits(rows, n, rank, dtype):
    """h next to the middle between what its bf16 numbers can hold: with nothing beside the adapter's part, and with a W x that takes all but its last bits away."""
    from paper_2605_22566_b200.runtime import Projection
    pa = _pa()
    x, a, b = (t.cuda() for t in D.between_numbers(rows, n, 3, rank))
    which = torch.arange(rows, dtype=torch.int32, device="cuda") % 4 - 1
    for w, ids in ((torch.zeros(n, 16, dtype=torch.bfloat16, device="cuda"), which), (D.cancelling(x.cpu(), b[1].cpu()).cuda(), torch.ones_like(which))):
        got = pa.project(Projection(w, a, b), x, ids, dtype=dtype).double()
        shared = x.double() @ w.double().T
        part = torch.zeros_like(shared)
        for i in range(3):
            mine = ids == i
            part[mine] = (x[mine].double() @ a[i].double().T) @ b[i].double().T
        ref = shared + part
        # (W x is one addition of 16 entries and one to what is there; its own digits are those of the row's magnitudes)
        bound = (D.THREE if dtype == torch.float32 else D.TWO) * part + 2 * 2.0 ** -23 * shared.abs() + torch.finfo(dtype).eps / 2 * ref.abs()
        assert bool(((got - ref).abs() <= bound).all()), float(((got - ref).abs() / (bound + 1e-300)).max())
    assert pa.status() == 0
    pa.close()


# ---- entries that are no numbers -------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,k,n,rank", [(5, 4096, 300, 8), (40, 264, 129, 16), (130, 1024, 700, 24), (100, 64, 20000, 16), (256, 2048, 600, 32), (300, 200, 100, 16), (700, 264, 520, 64),
                                           (2100, 128, 2500, 8)])
def test_an_adapter_that_is_no_number_spoils_its_own_rows_only(rows, k, n, rank, dtype):
    """Infinities and NaN in one adapter's B, one entry and all of it: other adapters' rows and rows without one are what they are without it, to rounding, its own what the formula
    gives.  (Written after the Projection was made, which refuses them.)"""
    from paper_2605_22566_b200.runtime import Projection
    rng = np.random.default_rng(rows + k)
    pa = _pa()
    x, w = _bf16(rng, rows, k).cuda(), (_bf16(rng, n, k) * k ** -0.5).cuda()
    a, b = (_bf16(rng, 5, rank, k) * k ** -0.5).cuda(), _bf16(rng, 5, n, rank).cuda()
    which = torch.from_numpy(rng.integers(-1, 5, rows)).to(torch.int32).cuda()
    which[0], which[-1] = 2, 3
    p = Projection(w, a, b)
    clean = pa.project(p, x, which, dtype=dtype)
    b[2, n // 2, rank - 1] = float("inf")
    b[2, 0, 0] = float("-inf")
    b[4, n - 1, 3] = float("nan")
    b[3] = float("nan")                                                 # every row of a tile that has one of this
    x[rows // 2, 1] = float("nan")
    got = pa.project(p, x, which, dtype=dtype)
    ok = (which != 3).cpu()
    ok[rows // 2] = False
    where = torch.arange(rows)
    ref, size = OS.project(*(t.double().cpu().numpy() for t in (x, w, a, b)), None, which.tolist())
    _, size = OS.project(*(t.double().cpu().nan_to_num(0.0, 0.0, 0.0).numpy() for t in (x, w, a, b)), None, which.tolist())
    y = got.double().cpu().numpy()
    bad = ~np.isfinite(ref)
    assert np.array_equal(np.isnan(y), np.isnan(ref)) and np.array_equal(y[bad & ~np.isnan(ref)], ref[bad & ~np.isnan(ref)])
    assert bad[~ok.numpy()].all() and bad[ok.numpy()].sum() == 2 * int((which[ok] == 2).sum()) + int((which[ok] == 4).sum())
    # (sums of k + rank products in fp32, in another order: 2^-23 of the magnitudes for each at most, twice for the adapter's; then half a step of the type)
    bound = 2 * (k + 80) * 2.0 ** -23 * size + np.abs(np.where(bad, 0.0, ref)) * torch.finfo(dtype).eps / 2
    assert np.all(np.abs(np.where(bad, 0.0, y) - np.where(bad, 0.0, ref)) <= bound * 1.001 + 1e-37)
    # tiles without such an adapter, and features without such an entry, have the same bits as before
    spoiled = {int(t) // 256 for t in where[(which == 3).cpu()]} | {rows // 2 // 256}
    same = [int(t) for t in where if int(t) // 256 not in spoiled and int(which[t]) not in (2, 4)]
    assert torch.equal(got[same], clean[same])
    none = pa.project(p, x, torch.full_like(which, -1), dtype=dtype)
    assert torch.equal(none[:rows // 2], pa.project(p, x, None, dtype=dtype)[:rows // 2])
    assert pa.status() == 0
    pa.close()


# ---- weights of tokens that took others' slots -------------------------------------------------------------


@pytest.mark.parametrize("captured", [False, True])
def test_weights_of_tokens_in_the_slots_of_tokens_taken_back(captured):
    """Steps of decode over open nodes that take tokens back, as after drafts that were not accepted: what every token has received is its own, and an
    eviction behind the last step goes by that."""
    rng = np.random.default_rng(2)
    hq, hkv, d, layers = 4, 2, 64, 2
    paths = [[0, 1], [0, 2], [0, 3]]
    pa = _pa([90, 150, 150, 150, 20], hq, hkv, d, layers, paths, extra_tiles=4)
    kv, mine = {}, {}
    for layer in range(layers):
        k, v = _bf16(rng, 90, hkv, d), _bf16(rng, 90, hkv, d)
        pa.write_node(0, layer, k.cuda(), v.cuda())
        kv[layer, 0] = [k.double().numpy(), v.double().numpy()]
        mine[layer, 0] = np.zeros((hkv, 90))
        for n in (1, 2, 3):
            kv[layer, n], mine[layer, n] = [np.zeros((0, hkv, d))] * 2, np.zeros((hkv, 0))
    for n in (1, 2, 3):
        pa.open_node(n, 150)
    weights = pa.new_weights()
    nodes = _ints(1, 2, 3)
    new = 90
    counts, held = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    k, v = (torch.zeros(layers, new, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(layers, 3, hq, d, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(layers, 3, hq, device="cuda")
    out = torch.empty_like(q)

    def step():
        slots, _ = pa.append_slots(nodes, counts, new, held)
        pa.clear_slot_weights(weights, slots)
        pa.build(deferred=True)
        for layer in range(layers):
            pa.append(layer, slots, k[layer], v[layer])
            pa.decode(layer, q[layer], out=out[layer], lse=lse[layer])
            pa.attention_weights(layer, q[layer], lse[layer], weights)
    graph = None
    pa.build(deferred=True)
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        assert pa.status() == 0
    for kept, more in (([0, 0, 0], [70, 1, 0]), ([70, 1, 0], [5, 2, 1]), ([71, 0, 1], [4, 1, 0]), ([60, 1, 1], [30, 0, 3]), ([90, 0, 2], [0, 0, 2])):
        held.copy_(_ints(*kept))
        counts.copy_(_ints(*more))
        for t in (k, v, q):
            t.copy_(_bf16(rng, *t.shape))
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        for layer in range(layers):
            begin = 0
            for i, n in enumerate((1, 2, 3)):
                rows = [t[layer, begin:begin + more[i]].double().cpu().numpy() for t in (k, v)]
                kv[layer, n] = [np.concatenate([old[:kept[i]], new_rows]) for old, new_rows in zip(kv[layer, n], rows)]
                mine[layer, n] = np.concatenate([mine[layer, n][:, :kept[i]], np.zeros((hkv, more[i]))], axis=1)
                begin += more[i]
            queries = q[layer].double().cpu().numpy()
            node_kv = lambda n: kv[layer, n]  # noqa: E731
            _, ref_lse = OA.decode(paths, node_kv, queries, hkv)
            for n, got in OE.attention_weights(paths, node_kv, queries, ref_lse, hkv).items():
                mine[layer, n] = mine[layer, n] + got
                held_now = weights[layer, :, pa.node_slot(n):pa.node_slot(n) + got.shape[1]].double().cpu().numpy()
                assert np.all(np.abs(held_now - mine[layer, n]) <= 2e-4 * mine[layer, n] + 1e-30), (layer, n)
        at = [a + b for a, b in zip(kept, more)]
    assert pa.status() == 0
    pa.close_node(1, at[0])
    before = weights.clone()
    kept_ids, = pa.evict([(4, 1, 20, 1, 1)], weights)
    for layer in range(layers):
        for h in range(hkv):
            slot = pa.node_slot(1)
            assert kept_ids[layer, h].tolist() == OE.kept(before[layer, h, slot:slot + at[0]].cpu().tolist(), 20, 1, 1)
    assert pa.status() == 0
    del graph
    pa.close()


def test_weights_are_cleared_where_new_tokens_are():
    pa = _pa([100, 64], 2, 2, 64, 2)
    weights = pa.new_weights()
    for slots, cleared in (([3, 70, 4, 3], {3, 4, 70}), ([-1, 5, -1], {5}), ([-1, -1], set()), ([0, -1], {0}), ([], set())):
        weights.fill_(1.5)
        pa.clear_slot_weights(weights, _ints(*slots))
        want = torch.full_like(weights, 1.5)
        want[:, :, sorted(cleared)] = 0
        assert torch.equal(weights, want), slots
    weights.fill_(float("nan"))
    pa.clear_slot_weights(weights, _ints(7, -1))
    assert bool((weights[:, :, 7] == 0).all()) and bool(weights[:, :, 0].isnan().all())
    for bad in (torch.tensor([1]), _ints(1).long(), _ints(1, 2)[::2].expand(2)):
        with pytest.raises(ValueError):
            pa.clear_slot_weights(weights, bad)
    with pytest.raises(ValueError):
        pa.clear_slot_weights(weights[:1], _ints(1))
    pa.close()


# ---- ids, and nodes that grow under an extend ----------------------------------------------------------------


@pytest.mark.parametrize("rows", [1, 300, 700])
def test_ids_of_a_projection_without_adapters_count_as_none_and_are_reported(rows):
    from paper_2605_22566_b200 import binding as B
    from paper_2605_22566_b200.runtime import Projection
    rng = np.random.default_rng(rows)
    pa = _pa()
    x, p = _bf16(rng, rows, 64).cuda(), Projection(_bf16(rng, 40, 64).cuda())
    want = pa.project(p, x, dtype=torch.float32)
    for last in (-1, 0, 5, -2, 2 ** 31 - 1):
        ids = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        ids[-1] = last
        y = torch.full_like(want, 7.0)
        assert B.gf_adapter_project(pa.g, p.desc, rows, x.data_ptr(), 64, ids.data_ptr(), y.data_ptr(), 40, 1, None, 0, pa.stream) == B.GF_OK
        assert torch.equal(y, want) and pa.status() == (B.GF_OK if last == -1 else B.GF_ERR_INVALID_ARG) and pa.status() == 0
    pa.close()


@pytest.mark.parametrize("d", [64, 128])
def test_extend_with_append_over_open_nodes(d):
    """Prompts that come into open nodes by the attention launch, at the length that the nodes have by then; zeros behind them, and growth goes on."""
    from paper_2605_22566_b200 import binding as B
    rng = np.random.default_rng(d)
    hq, hkv, layers = 4, 2, 2
    paths = [[0, 1], [0, 2], [3]]
    pa = _pa([70, 200, 130, 300], hq, hkv, d, layers, paths)
    pa.pool.fill_(0xFF)
    kv = {}
    for layer in range(layers):
        k, v = _bf16(rng, 70, hkv, d), _bf16(rng, 70, hkv, d)
        pa.write_node(0, layer, k.cuda(), v.cuda())
        kv[layer, 0] = (k.double().numpy(), v.double().numpy())
    for n, room in ((1, 200), (2, 130), (3, 300)):
        pa.open_node(n, room)
    lens = [65, 1, 129]
    pa.append_slots(_ints(1, 2, 3), _ints(*lens), sum(lens))
    pa.build(mode=B.GF_MODE_EXTEND)
    begin = np.concatenate([[0], np.cumsum(lens)])
    for layer in range(layers):
        q, k, v = _bf16(rng, sum(lens), hq, d), _bf16(rng, sum(lens), hkv, d), _bf16(rng, sum(lens), hkv, d)
        out = pa.extend_append(layer, q.cuda(), k.cuda(), v.cuda())
        for i, n in enumerate((1, 2, 3)):
            kv[layer, n] = tuple(t[begin[i]:begin[i + 1]].double().numpy() for t in (k, v))
        ref, _ = OA.extend(paths, lambda n: kv[layer, n], q.double().numpy(), hkv)
        assert_close(out.double().cpu().numpy(), ref, f"layer {layer}")
        assert torch.equal(pa.extend(layer, q.cuda()), out)               # (as over written nodes)
    slots, now = pa.append_slots(_ints(2, 1, 3), _ints(3, 0, 1), 4)
    assert now.tolist() == [4, 65, 130]
    k, v = _bf16(rng, 4, hkv, d), _bf16(rng, 4, hkv, d)
    for layer in range(layers):
        pa.append(layer, slots, k.cuda(), v.cuda())
        for n, rows in ((2, slice(0, 3)), (3, slice(3, 4))):
            kv[layer, n] = tuple(np.concatenate([a, b[rows].double().numpy()]) for a, b in zip(kv[layer, n], (k, v)))
        for n in (1, 2, 3):
            for got, want in zip(pa.load_node(n, layer), kv[layer, n]):
                got = got.double().cpu().numpy()
                assert np.array_equal(got[:len(want)], want) and not got[len(want):].any()
    one = torch.zeros(64, hkv, d, dtype=torch.bfloat16, device="cuda")
    assert B.gf_node_kv4_write(pa.g, 1, 0, one.data_ptr(), one.data_ptr(), 64, pa.stream) == B.GF_ERR_INVALID_ARG
    assert pa.status() == 0
    pa.close()


# ---- what lies beside results ----------------------------------------------------------------------------


def test_nothing_is_written_beside_results_and_scratch():
    """Results and scratch between bands of a pattern, of odd sizes; each band is looked at behind the calls."""
    from paper_2605_22566_b200.runtime import Projection
    rng = np.random.default_rng(3)
    pa = _pa([300] * 40, 2, 2, 64, 2)
    pa.guard_outputs = True
    for v in range(40):
        pa.open_node(v, 300)
    for n, more in ((1, 1), (7, 30), (40, 299)):
        slots, _ = pa.append_slots(_ints(*range(n)), torch.full((n,), more, dtype=torch.int32, device="cuda"), n * more + 3, torch.zeros(n, dtype=torch.int32, device="cuda"))
        rows = _bf16(rng, n * more + 3, 2, 64).cuda()
        pa.append(1, slots, rows, rows)
    for rows, k, n, adapters, rank in ((1, 64, 129, 3, 8), (77, 200, 999, 5, 24), (255, 128, 131, 70, 64), (300, 264, 100, 40, 16), (513, 72, 4099, 9, 32), (2100, 64, 257, 300, 8)):
        p = Projection((_bf16(rng, n, k) * 0.1).cuda(), (_bf16(rng, adapters, rank, k) * 0.1).cuda(), _bf16(rng, adapters, n, rank).cuda())
        ids = torch.from_numpy(rng.integers(-1, adapters, rows)).to(torch.int32).cuda()
        x = _bf16(rng, rows, k).cuda()
        for dtype in (torch.bfloat16, torch.float32):
            pa.project(p, x, ids, dtype=dtype)
            pa.project(p, x, None, dtype=dtype)
    for rows, v, top in ((1, 1, 1), (3, 70001, 32), (149, 999, 7), (2100, 130, 5)):
        for dtype in (torch.bfloat16, torch.float32):
            x = torch.from_numpy(rng.standard_normal((rows, v))).to(dtype).cuda()
            pa.token_logprobs(x, torch.zeros(rows, dtype=torch.int32, device="cuda"), top)
    assert len(pa._guards) > 60
    assert pa.status() == 0
    pa.verify_guards()
    pa.close()


def test_sizes_next_to_the_end_of_int32_are_refused_before_a_launch():
    from paper_2605_22566_b200 import binding as B
    pa = _pa()
    t = torch.zeros(1 << 12, device="cuda")
    p, most = t.data_ptr(), 2 ** 31 - 1
    for n in (2 ** 30 + 1, most):
        assert B.gf_append_slots(pa.g, n, p, None, p, 1, p, None, pa.stream) == B.gf_append_slots(pa.g, 1, p, None, p, n, p, None, pa.stream) == B.GF_ERR_INVALID_ARG
        assert B.gf_node_kv_append(pa.g, 0, n, p, p, 1024, p, 1024, pa.stream) == B.GF_ERR_INVALID_ARG
    for rows, out_dim in ((most, 8), (most - 510, 8), (1, most), (1, most - 510)):
        desc = B.ProjectionDesc(64, out_dim, p, 64, 0, 0, None, None, None)
        assert B.gf_adapter_project(pa.g, desc, rows, p, 64, None, p, out_dim, 1, None, 0, pa.stream) == B.GF_ERR_INVALID_ARG
    assert pa.status() == 0
    pa.close()
