"""Accumulated attention weights and eviction by them, against the fp64 definitions; and the operators in a row, as a serving
loop runs them."""
import numpy as np
import pytest
import torch

from helpers import assert_close
from kv4_cases import ODD_LENS, View, private_workload, random_case, two_stream_case
from oracle import attention as OA
from oracle import eviction as OE
from oracle import kv4
from oracle.residual import f64_to_bf16_rne
from paper_2605_22566_b200 import workloads as W

pytestmark = pytest.mark.gpu

# A weight is a sum of 2^x with x = scale log2(e) (sum of D products) - lse log2(e).  fp32 products are exact (bf16 by bf16), so
# x is off by the sum's roundings, at most (D + 8) 2^-24 sum |q k| scale log2(e): with |q|, |k| of unit spread the sum is about
# 0.64 D, which makes 136 * 2^-24 * 82 * 0.128 = 8.5e-5 for D = 128; lse in fp32 adds 1e-6 and ex2.approx 2^-22.
RTOL = 2e-4


def _handle(w, four=(), **kw):
    from paper_2605_22566_b200.runtime import PathAttention
    pa = PathAttention(w, kv4_nodes=four, **kw)
    pa.write_nodes("host")
    pa.build()
    return pa


def _reference(w, four, layer=0):
    view = View(w, four, layer)
    _, lse = OA.decode(view.paths(), view.node_kv, view.q(), w.num_kv_heads)
    return lse, OE.attention_weights(view.paths(), view.node_kv, view.q(), lse, w.num_kv_heads)


def _check_weights(pa, weights, ref, layer=0, factor=1.0, before=0.0, untouched=None):
    w = pa.w
    mine = torch.zeros(weights.shape[2], dtype=torch.bool)
    for v, want in ref.items():
        slot, n = pa.node_slot(v), int(w.node_len[v])
        mine[slot:slot + n] = True
        got = weights[layer, :, slot:slot + n].double().cpu().numpy()
        assert np.all(np.abs(got - (before + factor * want)) <= RTOL * (before + factor * want) + 1e-30), v
    rest = weights[layer][:, ~mine]
    assert bool((rest == (before if untouched is None else untouched)).all()), "a slot of no token on a path was written"


@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 64), (2, 1, 64), (16, 2, 64), (3, 3, 128), (4, 2, 128), (32, 8, 128), (8, 1, 128)])
@pytest.mark.parametrize("four", ["none", "all", "some"])
def test_weights_every_head_layout_and_odd_lengths(hq, hkv, d, four):
    w = random_case(hq, hkv, d, requests=9)
    nodes = {"none": [], "all": range(len(ODD_LENS)), "some": [v for v in range(len(ODD_LENS)) if v % 3 != 1]}[four]
    pa = _handle(w, nodes)
    lse, ref = _reference(w, nodes)
    q, l32 = pa.make_q(0, "host"), torch.from_numpy(lse.astype(np.float32)).cuda()
    weights = pa.new_weights()
    weights.fill_(0.25)
    pa.attention_weights(0, q, l32, weights, accumulate=True)
    _check_weights(pa, weights, ref, before=0.25)
    first = weights.clone()
    weights.fill_(0.25)
    pa.attention_weights(0, q, l32, weights, accumulate=True)
    assert torch.equal(weights, first)                       # a fixed order of additions
    weights.zero_()
    for _ in range(2):
        pa.attention_weights(0, q, l32, weights, accumulate=False)   # replaces
    _check_weights(pa, weights, ref)
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("requests", [5, 40])
@pytest.mark.parametrize("four", [[], [0, 2]])
def test_weights_of_a_later_layer_leave_the_others(requests, four):
    w = random_case(8, 2, 128, requests, lens=[300, 40, 129, 64], shared=0, layers=3)
    pa = _handle(w, four)
    weights = pa.new_weights()
    weights.fill_(0.5)
    for layer in (2, 1):
        lse, ref = _reference(w, four, layer)
        pa.attention_weights(layer, pa.make_q(layer, "host"), torch.from_numpy(lse.astype(np.float32)).cuda(), weights, accumulate=False)
        _check_weights(pa, weights, ref, layer, untouched=0.5)
    assert bool((weights[0] == 0.5).all())
    pa.close()


@pytest.mark.parametrize("requests", [1, 2, 40, 150])
@pytest.mark.parametrize("four", [[], [0, 2]])
def test_weights_of_widely_shared_nodes(requests, four):
    w = random_case(8, 2, 128, requests, lens=[700, 40, 129, 64], shared=0)
    pa = _handle(w, four)
    lse, ref = _reference(w, four)
    weights = pa.new_weights()
    pa.attention_weights(0, pa.make_q(0, "host"), torch.from_numpy(lse.astype(np.float32)).cuda(), weights)
    _check_weights(pa, weights, ref)
    pa.close()


def test_weights_more_segments_than_buckets():
    """Thousands of short segments: the tile search walks runs of segments."""
    n = 2500
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 90, n).tolist()
    w = private_workload(lens, [rng.permutation(n)[:25].tolist() for _ in range(100)], 2, 1, 64)
    pa = _handle(w, [v for v in range(n) if v % 2])
    lse, ref = _reference(w, [v for v in range(n) if v % 2])
    assert len(ref) > 1024
    weights = pa.new_weights()
    pa.attention_weights(0, pa.make_q(0, "host"), torch.from_numpy(lse.astype(np.float32)).cuda(), weights)
    _check_weights(pa, weights, ref)
    pa.close()


def test_weights_with_the_lse_of_decode_sum_to_the_heads_and_skip_residual_nodes():
    from paper_2605_22566_b200 import binding as B
    w = private_workload([200, 90, 64, 90], [[0, 2], [1, 2], [3], [0]], 8, 2, 128)
    pa = _handle(w, [0], max_residual_nodes=1)
    assert B.gf_node_kv_release(pa.g, 3, pa.stream) == B.GF_OK
    assert B.gf_node_kv_attach_residual(pa.g, 3, 0, 1, None, None, pa.stream) == B.GF_OK
    pa.build()
    q, lse = pa.make_q(0, "host"), torch.empty(4, 8, device="cuda")
    pa.decode(0, q, lse=lse)
    weights = pa.new_weights()
    pa.attention_weights(0, q, lse, weights)
    # requests 0, 1 and 3 give away 1 per head; request 2 attends to the residual node alone, which has no slots of its own
    assert abs(float(weights.sum()) - 3 * 8) < 24 * RTOL
    assert pa.status() == 0
    pa.close()


def test_weights_refusals():
    from paper_2605_22566_b200 import binding as B
    w = random_case(4, 2, 64, 3)
    pa = _handle(w)
    q, lse, weights = pa.make_q(0, "host"), torch.zeros(3, 4, device="cuda"), pa.new_weights()
    def call(**o):
        a = {**dict(layer=0, q=q.data_ptr(), lse=lse.data_ptr(), acc=1, w=weights.data_ptr()), **o}
        return B.gf_path_attention_weights(pa.g, pa.tables, a["layer"], a["q"], a["lse"], a["acc"], a["w"], pa.stream)
    assert call() == B.GF_OK
    assert call(layer=1) == call(q=None) == call(q=q.data_ptr() + 2) == call(lse=None) == call(w=None) == B.GF_ERR_INVALID_ARG
    assert call(w=weights.data_ptr() + 2) == call(acc=2) == B.GF_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        pa.attention_weights(0, q, lse, weights[:, :, :-1])
    with pytest.raises(ValueError):
        pa.attention_weights(0, q, lse.double(), weights)
    with pytest.raises(ValueError):
        pa.attention_weights(0, q.float(), lse, weights)
    assert B.gf_node_kv_release(pa.g, int(w.used_nodes()[0]), pa.stream) == B.GF_OK
    assert call() == B.GF_ERR_NOT_BUILT                       # tables are stale
    pa.close()


@pytest.mark.parametrize("four", [[], list(range(25)), [0, 2, 4]])
def test_weights_on_two_streams_captured_on_another_stream_and_deferred(four):
    """A batch whose two kernels run beside each other: against fp64, and the same bits from a call on another stream, from
    replayed graphs and from deferred tables; the slots of tokens that no path has stay as they were."""
    w = two_stream_case()
    pa = _handle(w, four, extra_tiles=2)
    q = pa.make_q(0, "host")
    lse, ref = _reference(w, four)
    lse = torch.from_numpy(lse.astype(np.float32)).cuda()
    weights = pa.new_weights()
    weights.fill_(-5.0)
    pa.attention_weights(0, q, lse, weights, accumulate=False)
    _check_weights(pa, weights, ref, untouched=-5.0)
    other = torch.full_like(weights, -5.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pa.attention_weights(0, q, lse, other, accumulate=False)
    side.synchronize()
    assert torch.equal(other, weights)
    twice = weights.clone()
    pa.attention_weights(0, q, lse, twice, accumulate=True)
    graph = torch.cuda.CUDAGraph()
    sums = weights.clone()
    with torch.cuda.graph(graph):
        pa.attention_weights(0, q, lse, sums, accumulate=True)
    for _ in range(2):
        sums.copy_(weights)
        graph.replay()
        assert torch.equal(sums, twice)
    pa.build(deferred=True)
    other.fill_(-5.0)
    pa.attention_weights(0, q, lse, other, accumulate=False)
    assert torch.equal(other, weights)
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("captured", [False, True])
def test_calls_at_once_behind_weights_on_two_streams(captured):
    """Weights that run on two streams, and behind them, without a wait, a decode into the very lse that they read and a build of
    the tables: nothing of what follows overtakes the second stream."""
    w = two_stream_case()
    pa = _handle(w, [0, 2, 4])
    q = pa.make_q(0, "host")
    other = torch.flip(q, [0]).contiguous()
    lse, out = torch.empty(40, 32, device="cuda"), torch.empty_like(q)
    wants = []
    for x in (q, other):                                      # one after the other
        pa.decode(0, x, out=out, lse=lse)
        torch.cuda.synchronize()
        weights = pa.new_weights()
        pa.attention_weights(0, x, lse, weights, accumulate=False)
        torch.cuda.synchronize()
        wants.append((lse.clone(), out.clone(), weights))
    got = [torch.zeros_like(wants[0][2]) for _ in wants]

    def run():
        for x, y in zip((q, other), got):
            pa.decode(0, x, out=out, lse=lse)
            pa.attention_weights(0, x, lse, y, accumulate=False)
        pa.decode(0, q, out=out, lse=lse)
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
    for _ in range(50):
        for y in got:
            y.zero_()
        if captured:
            graph.replay()
        else:
            run()
            pa.build()
        assert torch.equal(lse, wants[0][0]) and torch.equal(out, wants[0][1])
        assert all(torch.equal(y, want[2]) for y, want in zip(got, wants))
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("four", [False, True])
def test_a_new_node_on_the_slots_of_a_released_one_beside_an_old_node(four):
    """One batch with a node that has weights already and one that takes a released node's slots: cleared, the new one's are
    its own step's, and the old one's go on."""
    from paper_2605_22566_b200 import binding as B
    w = private_workload([100, 200, 130], [[0, 1], [0, 1], [0, 2]], 4, 2, 64)
    pa = _handle_unbuilt(w, range(3) if four else [])
    pa.write_nodes("host", only=[0, 1])
    pa.build()                                                 # (node 2 does not exist yet: an empty segment)
    q, lse, weights = pa.make_q(0, "host"), torch.empty(3, 4, device="cuda"), pa.new_weights()
    pa.decode(0, q, lse=lse)
    pa.attention_weights(0, q, lse, weights)
    slot, old = pa.node_slot(1), pa.node_weights(weights, 0).clone()
    assert float(pa.node_weights(weights, 1).sum()) > 1
    assert B.gf_node_kv_release(pa.g, 1, pa.stream) == B.GF_OK
    pa.write_nodes("host", only=[2])
    assert pa.node_slot(2) == slot and float(pa.node_weights(weights, 2).sum()) > 1      # the released node's sums
    pa.clear_node_weights(weights, 2)
    assert float(pa.node_weights(weights, 2).abs().sum()) == 0 and torch.equal(pa.node_weights(weights, 0), old)
    pa.build()
    pa.decode(0, q, lse=lse)
    alone = torch.zeros_like(weights)
    pa.attention_weights(0, q, lse, alone, accumulate=False)
    pa.attention_weights(0, q, lse, weights, accumulate=True)
    assert torch.equal(pa.node_weights(weights, 2), pa.node_weights(alone, 2))
    assert torch.equal(pa.node_weights(weights, 0), old + pa.node_weights(alone, 0))
    with pytest.raises(ValueError):
        pa.clear_node_weights(weights[:, :, :-1], 2)
    assert pa.status() == 0
    pa.close()


def test_weights_of_an_invalid_deferred_batch_change_nothing():
    from paper_2605_22566_b200 import binding as B
    w = private_workload([100, 64], [[0], [1]], 4, 2, 64)
    pa = _handle(w, [0])
    pa.path_node = torch.tensor([0, 7], dtype=torch.int32, device="cuda")
    pa.build(deferred=True)
    weights = torch.full_like(pa.new_weights(), 3.0)
    pa.attention_weights(0, pa.make_q(0, "host"), torch.zeros(2, 4, device="cuda"), weights)
    assert pa.status() == B.GF_ERR_INVALID_PATH
    assert bool((weights == 3.0).all())
    pa.close()


# ---- eviction -------------------------------------------------------------------------------------------


def _evict_case(lens, four, keeps, layers=2, hkv=2, d=64, first=0, last=0, make=None, seed=1):
    """Sources 0..n-1, destinations n..2n-1; checks indices, rows, zero tails, carried weights, untouched sources."""
    n = len(lens)
    w = private_workload(lens + [min(a, b) for a, b in zip(lens, keeps)], [[i] for i in range(2 * n)], hkv, hkv, d, layers=layers)
    pa = _handle_unbuilt(w, [v for v in range(2 * n) if four[v % n]])
    pa.write_nodes("host", only=[v for v in range(n) if lens[v] > 0])
    for v in range(n):
        if lens[v] == 0:
            pa.write_node(v, 0, *[torch.empty(0, hkv, d, dtype=torch.bfloat16, device="cuda")] * 2)
    rng = np.random.default_rng(seed)
    weights = pa.new_weights()
    given = []
    for v in range(n):
        x = (make(rng, (layers, hkv, lens[v])) if make else rng.random((layers, hkv, lens[v]))).astype(np.float32)
        given.append(x)
        pa.node_weights(weights, v).copy_(torch.from_numpy(x))
    kept = pa.evict([(n + v, v, keeps[v], first, last) for v in range(n)], weights)
    for v in range(n):
        m = min(lens[v], keeps[v])
        assert tuple(kept[v].shape) == (layers, hkv, m)
        idx = kept[v].cpu().numpy()
        got_w = pa.node_weights(weights, n + v).cpu().numpy()
        assert np.array_equal(pa.node_weights(weights, v).cpu().numpy(), given[v], equal_nan=True)
        for layer in range(layers):
            src, dst = pa.load_node(v, layer), pa.load_node(n + v, layer)
            for h in range(hkv):
                want = OE.kept(given[v][layer, h], keeps[v], first, last)
                assert idx[layer, h].tolist() == want, (v, layer, h)
                assert np.array_equal(got_w[layer, h], given[v][layer, h][want], equal_nan=True)
                for s, t in zip(src, dst):
                    assert torch.equal(s[want, h].view(torch.int16), t[:, h].view(torch.int16)), (v, layer, h)
    assert pa.status() == 0
    return pa, weights


def _handle_unbuilt(w, four, **kw):
    from paper_2605_22566_b200.runtime import PathAttention
    return PathAttention(w, kv4_nodes=four, **kw)


@pytest.mark.parametrize("hkv,d", [(2, 64), (1, 128), (3, 128)])
@pytest.mark.parametrize("four", [False, True])
def test_evict_odd_lengths(hkv, d, four):
    lens = [1, 16, 63, 64, 65, 200, 130, 0]
    keeps = [1, 5, 63, 30, 64, 129, 1, 4]
    pa, _ = _evict_case(lens, [four] * 8, keeps, hkv=hkv, d=d)
    pa.close()


@pytest.mark.parametrize("first,last,keeps", [(0, 0, [0, 7, 300]), (4, 32, [40, 36, 300]), (0, 5, [5, 5, 5]), (64, 64, [128, 200, 257]), (3, 5, [129, 64, 128]), (1, 1, [128, 36, 127])])
def test_evict_protected_ends_and_both_kinds(first, last, keeps):
    pa, _ = _evict_case([257, 100, 300], [True, False, True], keeps, first=first, last=last)
    pa.close()


def _ties(rng, shape):
    return rng.integers(0, 4, shape) / 4.0


def _special(rng, shape):
    x = rng.standard_normal(shape) * 10.0 ** rng.integers(-40, 38, shape)
    pick = rng.integers(0, 12, shape)
    for i, s in enumerate([np.nan, np.inf, -np.inf, -0.0, 0.0]):
        x[pick == i] = s
    return x


@pytest.mark.parametrize("make", [_ties, _special, lambda r, s: np.zeros(s), lambda r, s: np.full(s, np.nan)])
def test_evict_ties_and_special_weights(make):
    pa, _ = _evict_case([513, 64, 2100], [False, True, True], [200, 33, 1111], make=make, first=1, last=2)
    pa.close()


def test_evict_a_long_node_and_many_entries():
    pa, _ = _evict_case([9000], [True], [4097], layers=1, hkv=1)
    pa.close()
    lens = [10 + v for v in range(40)]                                 # more entries than one launch takes
    pa, _ = _evict_case(lens, [v % 2 == 0 for v in range(40)], [5 + v // 2 for v in range(40)], layers=1, hkv=1)
    pa.close()


@pytest.mark.parametrize("make", [None, _ties, _special, lambda r, s: np.full(s, np.nan)])
def test_evict_around_the_longest_held_in_registers(make):
    pa, _ = _evict_case([8191, 8192, 8193, 20000], [True, False, True, True], [8190, 4095, 1, 20000], layers=1, hkv=1, make=make, last=1)
    pa.close()


def test_evict_twice_into_the_same_node_and_one_source_into_two():
    pa, weights = _evict_case([150], [False], [70])
    again = pa.node_weights(weights, 0)
    again.copy_(again.flip(2))
    (kept,) = pa.evict([(1, 0, 70, 0, 0)], weights)
    for layer in range(2):
        for h in range(2):
            assert kept[layer, h].tolist() == OE.kept(again[layer, h].cpu().numpy(), 70, 0, 0)
    pa.close()


def _tail_of_4_bit_part(part, d, values, first):
    """The codes and (s, lo) words of a 4-bit tile's K (values False) or V part that belong to tokens from `first` on (the layout
    of kv4_device.cuh)."""
    groups = d // 64
    words = part[:32 * d].view(np.uint32).reshape(4, groups, 32, 4)          # [block of 16, group, lane, word]
    b, lane, nibble = np.arange(4)[:, None, None], np.arange(32)[:, None], np.arange(8)
    half, j, l4, l8 = nibble // 4, nibble % 4, lane % 4, lane // 4
    token = 16 * b + (2 * l4 + half + 8 * (j // 2) if values else l8 + 8 * (j % 2) + 0 * half)
    codes = words[..., None] >> (16 * half + 4 * j).astype(np.uint32) & 15   # [block, group, lane, word, nibble]
    at = np.broadcast_to(token[:, None, :, None, :], codes.shape) >= first
    return np.concatenate([codes[at], part[32 * d:].view(np.uint32).reshape(64, groups)[first:].ravel()])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("n,m", [(1, 1), (70, 7), (150, 33), (300, 177), (500, 64)])
def test_rows_behind_the_last_token_are_zeros(d, four, n, m):
    """Pools full of NaN patterns: the last tile of a written node (n tokens) and of an evicted one (m of them; in one launch and in
    two) holds zeros behind the last token, in every layer and head; attention multiplies them by 0."""
    hkv, layers = 3, 2
    w = private_workload([n, m], [[0], [1]], hkv, hkv, d, layers=layers)
    pa = _handle_unbuilt(w, [0, 1] if four else [])
    pool = pa.pool4 if four else pa.pool
    pool.fill_(0xFF)
    pa.write_nodes("host", only=[0])
    weights = pa.new_weights()
    pa.node_weights(weights, 0).copy_(torch.rand(layers, hkv, n, generator=torch.Generator().manual_seed(n)))
    pa.evict([(1, 0, m, 0, 0)], weights)
    from paper_2605_22566_b200 import binding as B
    info, size = (B.gf_kv4_pool_info(pa.g), B.gf_kv4_bytes_per_tile(d)) if four else (B.gf_pool_info(pa.g), B.gf_pool_bytes_per_tile(d))
    tiles = pool.cpu().numpy()[:layers * hkv * info.capacity_tiles * size].reshape(layers * hkv, info.capacity_tiles, size)
    before = 0 if not four else B.gf_pool_info(pa.g).capacity_tiles
    for node, count in ((0, n), (1, m)):
        last, rows = pa.node_slot(node) // 64 - before + (count - 1) // 64, (count - 1) % 64 + 1
        for tile in tiles[:, last]:
            if four:
                parts = [_tail_of_4_bit_part(part, d, i == 1, rows) for i, part in enumerate(tile.reshape(2, size // 2))]
                assert sum(map(len, parts)) == 2 * (64 - rows) * (d + d // 64) and not np.concatenate(parts).any()
            else:
                assert not tile.reshape(2 * d // 64, 64, 128)[:, rows:].any()
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("four", [False, True])
def test_evict_one_source_into_two_nodes(four):
    w = private_workload([200, 70, 129], [[0], [1], [2]], 2, 2, 64)
    pa = _handle_unbuilt(w, range(3) if four else [])
    pa.write_nodes("host", only=[0])
    weights = pa.new_weights()
    pa.node_weights(weights, 0).copy_(torch.rand(1, 2, 200, generator=torch.Generator().manual_seed(3)))
    given = pa.node_weights(weights, 0)[0].cpu().numpy()
    kept = pa.evict([(1, 0, 70, 3, 0), (2, 0, 129, 0, 8)], weights)
    for node, m, first, last in ((1, 70, 3, 0), (2, 129, 0, 8)):
        for h in range(2):
            want = OE.kept(given[h], m, first, last)
            assert kept[node - 1][0, h].tolist() == want
            assert np.array_equal(pa.node_weights(weights, node)[0, h].cpu().numpy(), given[h][want])
            for src, dst in zip(pa.load_node(0, 0), pa.load_node(node, 0)):
                assert torch.equal(src[want, h], dst[:, h])
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("keep", [100, 700])
def test_evict_captured_and_on_another_stream(four, keep):
    """Into a node that exists: a replayed graph chooses by the weights of the moment, as the plain call does."""
    w = private_workload([900, keep], [[0], [1]], 2, 2, 128)
    pa = _handle_unbuilt(w, [0, 1] if four else [])
    pa.write_nodes("host", only=[0])
    weights = pa.new_weights()
    (first,) = pa.evict([(1, 0, keep, 2, 5)], weights)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        (kept,) = pa.evict([(1, 0, keep, 2, 5)], weights)
    side = torch.cuda.Stream()
    for seed in (1, 2):
        pa.node_weights(weights, 0).copy_(torch.rand(1, 2, 900, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        got = kept.clone(), pa.node_weights(weights, 1).clone(), *pa.load_node(1, 0)
        for h in range(2):
            assert got[0][0, h].tolist() == OE.kept(pa.node_weights(weights, 0)[0, h].cpu().numpy(), keep, 2, 5)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            (again,) = pa.evict([(1, 0, keep, 2, 5)], weights)
            new = again, pa.node_weights(weights, 1), *pa.load_node(1, 0)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, new))
    assert pa.status() == 0
    pa.close()


def test_evict_refusals_change_nothing():
    from paper_2605_22566_b200 import binding as B
    w = private_workload([100, 64, 30, 40, 100], [[0], [1]], 2, 2, 64)
    pa = _handle_unbuilt(w, [1], extra_tiles=1, extra_kv4_tiles=1)
    pa.write_nodes("host", only=[0, 1])
    pa.build()
    weights, kept = pa.new_weights(), torch.zeros(4096, dtype=torch.int32, device="cuda")
    def evict(*entries, w=weights.data_ptr(), k=kept.data_ptr()):
        return B.gf_node_kv_evict(pa.g, entries, w, k, pa.stream)
    bad = B.GF_ERR_INVALID_ARG
    assert evict() == B.GF_OK
    assert evict((0, 0, 5, 0, 0)) == bad                                # a node into itself
    assert evict((2, 0, 5, 0, 0), (2, 1, 5, 0, 0)) == bad              # two states for one node
    assert evict((2, 0, 5, 0, 0), (3, 2, 5, 0, 0)) in (bad, B.GF_ERR_NOT_WRITTEN)
    assert evict((2, 0, 5, 3, 3)) == evict((2, 0, -1, 0, 0)) == evict((2, 0, 5, -1, 0)) == evict((9, 0, 5, 0, 0)) == evict((2, -1, 5, 0, 0)) == bad
    assert evict((2, 0, 5, 0, 0), w=None) == evict((2, 0, 5, 0, 0), k=None) == evict((2, 0, 5, 0, 0), w=weights.data_ptr() + 1) == bad
    assert evict((2, 3, 5, 0, 0)) == B.GF_ERR_NOT_WRITTEN
    assert evict((1, 0, 64, 0, 0)) == bad                               # written already, in the other pool
    before = B.gf_pool_info(pa.g).tiles_in_use, B.gf_kv4_pool_info(pa.g).tiles_in_use
    assert evict((2, 0, 30, 0, 0), (3, 1, 40, 0, 0), (4, 0, 100, 0, 0)) == B.GF_ERR_CAPACITY
    assert before == (B.gf_pool_info(pa.g).tiles_in_use, B.gf_kv4_pool_info(pa.g).tiles_in_use)
    assert B.gf_node_extent(pa.g, 2)[0] == B.gf_node_extent(pa.g, 3)[0] == B.GF_ERR_NOT_WRITTEN
    q = pa.make_q(0, "host")
    pa.decode(0, q)                                                       # the tables are still good
    assert not kept.any() and pa.status() == 0
    assert evict((2, 0, 30, 0, 0), (3, 1, 40, 0, 0)) == B.GF_OK          # and now it fits
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("four", [False, True])
def test_a_serving_loop_decode_weigh_evict_decode(four):
    """Three steps' weights, the shared node cut to a half, and decode over paths that name the cut node, all against fp64."""
    lens, n_req, m = [400, 60, 33, 17, 50], 4, 200
    paths = [[0, 1 + r % 4] for r in range(n_req)]
    nodes = list(range(6)) if four else []
    w = private_workload(lens + [m], paths + [[5]], 8, 2, 128)
    pa = _handle_unbuilt(w, nodes)
    pa.write_nodes("host", only=range(5))
    pa.build()
    view = View(w, nodes)
    weights, total = pa.new_weights(), 0.0
    ppl = [[v for v in p if v != 5] for p in view.paths()]
    for step in range(3):
        q = torch.roll(pa.make_q(0, "host"), step, 0).contiguous()
        lse = torch.empty(n_req + 1, 8, device="cuda")
        pa.decode(0, q, lse=lse)
        pa.attention_weights(0, q, lse, weights, accumulate=step > 0)
        qd = np.roll(view.q(), step, 0)
        _, ref_lse = OA.decode(ppl[:n_req], view.node_kv, qd[:n_req], 2)
        total = total + OE.attention_weights(ppl[:n_req], view.node_kv, qd[:n_req], ref_lse, 2)[0]
    got = pa.node_weights(weights, 0)[0].double().cpu().numpy()
    assert np.all(np.abs(got - total) <= 10 * RTOL * total)     # lse of decode is itself within 2e-3
    (kept,) = pa.evict([(5, 0, m, 4, 32)], weights)
    idx = kept[0].cpu().numpy()
    for h in range(2):
        assert idx[h].tolist() == OE.kept(got[h].astype(np.float32), m, 4, 32)
    # the same batch with the cut node in the place of node 0
    new = torch.tensor(sum([[5 if v == 0 else v for v in p] for p in paths], []) + [5], dtype=torch.int32, device="cuda")
    pa.path_node = new
    pa.build()
    q = pa.make_q(0, "host")
    out = pa.decode(0, q)
    K, V = view.node_kv(0)
    cut = tuple(np.stack([x[idx[h], h] for h in range(2)], 1) for x in (K, V))
    ref, _ = OA.decode([[5, p[1]] for p in paths] + [[5]], lambda v: cut if v == 5 else view.node_kv(v), view.q(), 2)
    assert_close(out.double().cpu().numpy(), ref, "decode over the cut node")
    assert pa.status() == 0
    pa.close()
