"""Node states held in 4 bits: what is stored against the definition, and decode over them against fp64 attention over the
values that the codes stand for."""
import numpy as np
import pytest
import torch

from helpers import assert_close
from kv4_cases import ODD_LENS, View, private_workload, random_case, two_stream_case
from oracle import attention as OA
from oracle import kv4
from oracle.residual import bf16_to_f64, f64_to_bf16_rne
from paper_2605_22566_b200 import workloads as W

pytestmark = pytest.mark.gpu


def _handle(w, four, **kw):
    from paper_2605_22566_b200.runtime import PathAttention
    return PathAttention(w, kv4_nodes=four, **kw)


def _bits(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


_bf16 = kv4.round_to_bf16


def _tensor(x):
    """bf16 numbers in fp64 as a tensor."""
    return torch.from_numpy((x.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16).view(np.int16)).cuda().view(torch.bfloat16)


# ---- storage --------------------------------------------------------------------------------------


@pytest.mark.parametrize("hkv,d", [(1, 64), (3, 64), (8, 128), (2, 128)])
def test_stored_values_bit_for_bit(hkv, d):
    lens = [1, 15, 16, 17, 64, 65, 200]
    w = private_workload(lens, [[i] for i in range(len(lens))], hkv, hkv, d, layers=2)
    pa = _handle(w, range(len(lens)))
    pa.write_nodes("host")
    for layer in (0, 1):
        for v, n in enumerate(lens):
            for got, bits in zip(pa.load_node(v, layer), w.node_kv_bits(layer, v)):
                want = f64_to_bf16_rne(kv4.values(W.bf16_bits_to_f64(bits)))
                assert np.array_equal(_bits(got), want), (layer, v)
    assert pa.status() == 0
    pa.close()


def test_stored_values_next_to_a_border_of_two_cells():
    """Entries within an fp32 step of a whole number of cells above lo: x - lo rounded to fp32 decides."""
    x = np.zeros((4, 1, 64))
    x[:, 0, 0], x[:, 0, 1] = -4.0, 4.0                     # s = 1/2: cells begin at every half
    tiny = 2.0 ** np.arange(-30, -8)
    x[0, 0, 2:24], x[1, 0, 2:24], x[2, 0, 2:24], x[3, 0, 2:24] = tiny, -tiny, 1 - tiny, -2.5 - tiny
    x = _bf16(x)
    w = private_workload([4], [[0]], 1, 1, 64)
    pa = _handle(w, [0])
    t = _tensor(x)
    pa.write_node(0, 0, t, t)
    for got in pa.load_node(0, 0):
        assert np.array_equal(_bits(got), f64_to_bf16_rne(kv4.values(x)))
    pa.close()


@pytest.mark.parametrize("exponent", [0, -100, 90])
def test_stored_values_next_to_a_border_are_those_of_the_exact_quotient(exponent):
    """Entries closer to a border of two cells than fp32 can tell beside lo: those below it lie in the lower cell."""
    tiny = 2.0 ** -np.arange(10.0, 31)
    x = np.zeros((4, 1, 64))
    x[:, 0, 0], x[:, 0, 1] = -4.0, 4.0                     # s = 1/2
    x[0, 0, 2:23], x[1, 0, 2:23] = tiny, -tiny
    x[2, 0, 0], x[2, 0, 2] = -2.0 ** -30, 0.25             # s = 1/4; lo just below 0, then just above
    x[3, 0, 0], x[3, 0, 2], x[3, 0, 3:] = 2.0 ** -30, 0.25, 2.0 ** -30
    x *= 2.0 ** exponent
    pa = _handle(private_workload([4], [[0]], 1, 1, 64), [0])
    t = _tensor(_bf16(x))
    pa.write_node(0, 0, t, t)
    want = np.concatenate([np.full(21, 0.25), np.full(21, -0.25), [1.5 * 0.25, 0.5 * 0.25]]) * 2.0 ** exponent
    for got in pa.load_node(0, 0):
        got = bf16_to_f64(_bits(got))[:, 0]
        assert np.array_equal(np.concatenate([got[0, 2:23], got[1, 2:23], [got[2, 2], got[3, 2]]]), want)
    pa.close()


@pytest.mark.parametrize("scale", [1e-35, 1.0, 2e36])
def test_stored_values_of_unusual_groups(scale):
    """Constant groups, one outlier, a spread far below the values, tiny and huge entries.  A value is computed in fp32 and
    rounded to bf16: within half a bf16 step (2^-8) and half an fp32 step (2^-24) of the definition's."""
    rng = np.random.default_rng(7)
    x = rng.standard_normal((70, 2, 128))
    x[0] = 0.75
    x[1, 0, :64] = 0.0
    x[2, 1, 5] = 90.0
    x[3] = 64.0 + 0.5 * rng.integers(0, 3, (2, 128))
    x[4] = -np.abs(x[4])
    x = _bf16(x * scale)
    w = private_workload([70], [[0]], 2, 2, 128)
    pa = _handle(w, [0])
    t = _tensor(x)
    pa.write_node(0, 0, t, t)
    want = kv4.values(x)
    for got in pa.load_node(0, 0):
        got = bf16_to_f64(_bits(got))
        assert np.all(np.abs(got - want) <= np.abs(want) * (2.0 ** -8 + 2.0 ** -23))
    pa.close()


def test_largest_finite_range_does_not_overflow():
    big = float(torch.finfo(torch.bfloat16).max)
    x = np.zeros((3, 1, 64))
    x[:, :, ::2], x[:, :, 1::2] = big, -big
    w = private_workload([3], [[0]], 1, 1, 64)
    pa = _handle(w, [0])
    t = _tensor(x)
    pa.write_node(0, 0, t, t)
    k, v = pa.load_node(0, 0)
    want = kv4.values(x)
    assert np.all(np.isfinite(want))
    for got in (k, v):
        assert np.all(np.abs(bf16_to_f64(_bits(got)) - want) <= np.abs(want) * (2.0 ** -8 + 2.0 ** -23))
    pa.close()


def test_stored_values_of_the_smallest_groups():
    """Groups whose entries differ by 2^-118 down to the subnormals' step 2^-133: s has no reciprocal in fp32 from 2^-124 on,
    and is a subnormal itself, or 0, further down.  Differences of such entries are exact in fp32, and so is every value."""
    rng = np.random.default_rng(19)
    steps = np.concatenate([np.arange(17), rng.integers(-16, 17, 47)])          # whole numbers of up to 16: exact in bf16
    x = np.stack([np.stack([rng.permutation(steps), 128 + rng.permutation(np.arange(64) % 17)]) * 2.0 ** -e for e in range(118, 134)])
    x[12:, 1] = np.abs(x[12:, 0])                                                # (the others there would not be small any more)
    x[15, 1] = rng.integers(0, 6, 64) * 2.0 ** -133                              # s is 0, the entries are not equal
    x = _bf16(x.reshape(-1, 1, 64))
    n = len(x)
    pa = _handle(private_workload([n], [[0]], 1, 1, 64), [0])
    t = _tensor(x)
    pa.write_node(0, 0, t, t)
    _, s, _ = kv4.encode(x)
    assert s.max() < 2.0 ** -115 and (s == 0).any() and ((s > 0) & (s < 2.0 ** -126)).any()
    want = _bf16(kv4.values(x))
    for got in pa.load_node(0, 0):
        assert np.array_equal(bf16_to_f64(_bits(got)), want)
    pa.close()


@pytest.mark.parametrize("value", [1e30, -3.0, 2.0 ** -130])
def test_constant_groups_of_any_size_are_exact(value):
    x = _bf16(np.full((20, 2, 64), value))
    pa = _handle(private_workload([20], [[0]], 2, 2, 64), [0])
    t = _tensor(x)
    pa.write_node(0, 0, t, t)
    assert all(torch.equal(got, t) for got in pa.load_node(0, 0))
    pa.close()


def test_extents_release_rewrite_and_refusals():
    from paper_2605_22566_b200 import binding as B
    w = private_workload([100, 64, 30, 0, 100, 10], [[0], [1], [2]], 2, 2, 64)
    pa = _handle(w, [0, 1], extra_tiles=1)      # 4-bit pool: 3 tiles; bf16 pool: 2
    buf = torch.randn(128, 2, 64, device="cuda").to(torch.bfloat16)
    p, s = buf.data_ptr(), pa.stream
    cap16 = B.gf_pool_info(pa.g).capacity_tiles
    assert B.gf_kv4_pool_info(pa.g).capacity_tiles == 3
    assert B.gf_node_kv4_write(pa.g, 0, 0, p, p, 100, s) == B.GF_OK
    assert B.gf_node_extent(pa.g, 0) == (B.GF_OK, 100, cap16 * 64)
    assert B.gf_node_kv4_write(pa.g, 1, 0, p, p, 64, s) == B.GF_OK
    assert B.gf_node_extent(pa.g, 1) == (B.GF_OK, 64, cap16 * 64 + 128)
    assert B.gf_weight_slots(pa.g) == (cap16 + 3) * 64
    assert B.gf_node_kv4_write(pa.g, 4, 0, p, p, 1, s) == B.GF_ERR_CAPACITY
    assert B.gf_node_kv4_write(pa.g, 0, 0, p, p, 99, s) == B.GF_ERR_INVALID_ARG      # another length
    assert B.gf_node_kv4_write(pa.g, 0, 0, p + 2, p, 100, s) == B.GF_ERR_INVALID_ARG  # alignment
    assert B.gf_node_kv4_write(pa.g, 0, 1, p, p, 100, s) == B.GF_ERR_INVALID_ARG     # no such layer
    assert B.gf_node_kv_write(pa.g, 0, 0, p, p, 100, s) == B.GF_ERR_INVALID_ARG      # held in 4 bits
    assert B.gf_node_kv_reserve(pa.g, 0, 100, s) == B.GF_ERR_INVALID_ARG
    assert B.gf_node_kv_write(pa.g, 2, 0, p, p, 30, s) == B.GF_OK
    assert B.gf_node_kv4_write(pa.g, 2, 0, p, p, 30, s) == B.GF_ERR_INVALID_ARG      # held in bf16
    assert B.gf_node_kv_reconstruct(pa.g, 4, 0, 0, None, None, s) == B.GF_ERR_INVALID_ARG
    assert B.gf_node_kv_attach_residual(pa.g, 4, 0, 0, None, None, s) == B.GF_ERR_INVALID_ARG
    assert B.gf_residual_encode(pa.g, 0, 0, p, p, 0.0, None, None, s) == B.GF_ERR_INVALID_ARG
    assert B.gf_kv4_pool_attach(pa.g, pa.pool4.data_ptr(), pa.pool4.numel()) == B.GF_ERR_INVALID_ARG  # nodes in it
    assert B.gf_node_kv4_write(pa.g, 3, 0, None, None, 0, s) == B.GF_OK              # an empty node has no tiles
    assert B.gf_node_kv_read(pa.g, 3, 0, None, None, s) == B.GF_OK
    assert B.gf_node_kv_release(pa.g, 0, s) == B.GF_OK
    assert B.gf_kv4_pool_info(pa.g).tiles_in_use == 1
    assert B.gf_node_kv4_write(pa.g, 5, 0, p, p, 10, s) == B.GF_OK                   # takes the hole's first tile
    assert B.gf_node_extent(pa.g, 5) == (B.GF_OK, 10, cap16 * 64)
    assert B.gf_node_kv_write(pa.g, 0, 0, p, p, 30, s) == B.GF_OK                    # and node 0 may be held in bf16 now
    for v in (1, 3, 5):
        assert B.gf_node_kv_release(pa.g, v, s) == B.GF_OK
    info = B.gf_kv4_pool_info(pa.g)
    assert (info.tiles_in_use, info.high_water_tiles) == (0, 0)
    assert B.gf_kv4_pool_attach(pa.g, pa.pool4.data_ptr() + 16, pa.pool4.numel()) == B.GF_ERR_INVALID_ARG
    assert B.gf_kv4_pool_attach(pa.g, pa.pool4.data_ptr(), 64) == B.GF_ERR_CAPACITY
    assert B.gf_kv4_pool_attach(pa.g, pa.pool4.data_ptr(), pa.pool4.numel()) == B.GF_OK
    assert pa.status() == 0
    with pytest.raises(ValueError):
        pa.write_node(1, 0, buf.float(), buf.float())
    with pytest.raises(ValueError):
        pa.write_node(1, 0, buf[:, :, :32], buf[:, :, :32])
    pa.close()


def test_a_handle_without_a_4_bit_pool_refuses():
    from paper_2605_22566_b200 import binding as B
    w = private_workload([10], [[0]], 2, 2, 64)
    pa = _handle(w, [])
    buf = torch.zeros(10, 2, 64, dtype=torch.bfloat16, device="cuda")
    assert B.gf_node_kv4_write(pa.g, 0, 0, buf.data_ptr(), buf.data_ptr(), 10, pa.stream) == B.GF_ERR_CAPACITY
    assert B.gf_kv4_pool_info(pa.g).capacity_tiles == 0
    pa.close()


# ---- decode ---------------------------------------------------------------------------------------------


def _decode(w, four, policy=None, deferred=False, check=True, source="host"):
    from paper_2605_22566_b200.runtime import tensor_to_f64
    pa = _handle(w, four, policy=policy)
    pa.write_nodes(source)
    pa.build(deferred=deferred)
    q = pa.make_q(0, source)
    lse = pa.guarded(w.num_requests * w.num_q_heads * 4, "lse").view(torch.float32).view(w.num_requests, w.num_q_heads)
    out = pa.decode(0, q, lse=lse)
    assert pa.status() == 0
    got, got_lse = tensor_to_f64(out), tensor_to_f64(lse)
    if check:
        view = View(w, four)
        ref, ref_lse = OA.decode(view.paths(), view.node_kv, view.q(), w.num_kv_heads)
        assert_close(got, ref, "out")
        seen = np.isfinite(ref_lse)
        assert np.array_equal(np.isneginf(got_lse), ~seen)
        assert np.abs(got_lse[seen] - ref_lse[seen]).max() < 2e-3
    pa.close()
    return got, got_lse


@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 64), (2, 1, 64), (8, 2, 64), (16, 2, 64), (3, 3, 128), (4, 2, 128), (32, 8, 128), (8, 1, 128)])
@pytest.mark.parametrize("four", ["all", "some"])
def test_decode_every_head_layout_and_odd_lengths(hq, hkv, d, four):
    w = random_case(hq, hkv, d, requests=9)
    _decode(w, range(len(ODD_LENS)) if four == "all" else [v for v in range(len(ODD_LENS)) if v % 3 != 1])


@pytest.mark.parametrize("requests", [1, 3, 16, 17, 70])
def test_decode_shared_by_few_and_many(requests):
    """One to many 16-row groups per item, more requests than one item takes, every node shared."""
    w = random_case(8, 2, 128, requests, lens=[300, 40, 129, 64], shared=0)
    _decode(w, range(4))


@pytest.mark.parametrize("policy", [(64, 1, 1, 1), (64, 3, 1, 2), (128, 16, 16, 4), (1024, 7, 2, 16)])
@pytest.mark.parametrize("deferred", [False, True])
def test_decode_policies(policy, deferred):
    w = random_case(8, 2, 128, 20, lens=[700, 40, 129, 64, 333], shared=0)
    _decode(w, [0, 2, 3], policy=policy, deferred=deferred)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64)])
def test_decode_one_request_over_many_chunks(hq, hkv, d):
    """Few rows with over 32 partial slots each: the merge shares them among eight warps."""
    w = private_workload([6000, 3001, 70], [[0, 1, 2], [1]], hq, hkv, d)
    _decode(w, [0, 1], policy=(64, 4, 1, 1))
    _decode(w, [0], policy=(64, 4, 1, 1), deferred=True)


@pytest.mark.parametrize("cfg,frac", [(1, 0.5), (3, 0.5), (3, 1.0)])
def test_decode_beside_the_tensor_memory_kernel(cfg, frac):
    """Batches whose widely shared bf16 segments run on the side stream, while others are held in 4 bits: two reduced configurations."""
    over = dict(n_requests=150, n_nodes=40, root_len=2500, len_lo=20, len_hi=300, suffix_max=60)
    w = W.make_config(cfg, **over)
    used = w.used_nodes()
    rng = np.random.default_rng(4)
    four = [int(v) for v in used if v != 0 and rng.random() < frac] + ([0] if frac == 1.0 else [])
    _decode(w, four, source="device")


@pytest.mark.parametrize("q_log2", [3, 5])
def test_decode_peaked_scores(q_log2):
    """Queries scaled up and planted keys: the running maximum moves late in the walk; scores reach hundreds."""
    w = random_case(8, 2, 128, 5, lens=[400, 200, 100, 64], shared=0, q_scale_log2=q_log2, v_scale_log2=-2,
                    planted=((0, 1, 0, 390, -1), (2, 6, 0, 170, -1), (4, 3, 0, 70, -1)))
    _decode(w, range(4))


def test_decode_large_and_tiny_value_scales():
    """Values whose groups differ by 2^40 in size between tokens: a small token that carries the weight is not drowned by
    a large one that carries none."""
    d, n = 128, 100
    rng = np.random.default_rng(11)
    k = rng.standard_normal((n, 1, d)) * 0.1
    q = rng.standard_normal((1, 1, d)) * 4
    k[50] = q[0] * 8          # nearly all of the weight
    v = rng.standard_normal((n, 1, d))
    v[7] *= 2.0 ** 20
    v[50] *= 2.0 ** -20
    k, q, v = _bf16(k), _bf16(q), _bf16(v)
    w = private_workload([n], [[0]], 1, 1, d)
    pa = _handle(w, [0])
    pa.write_node(0, 0, _tensor(k), _tensor(v))
    pa.build()
    out = pa.decode(0, _tensor(q)).double().cpu().numpy()
    ref, _ = OA.decode([[0]], lambda _: (kv4.values(k), kv4.values(v)), q, 1)
    assert pa.status() == 0
    # one rounding of p to bf16 (2^-8) per term and the output's (2^-8), against the largest output of the head
    assert np.abs(out - ref).max() <= 2.0 ** -7 * np.abs(ref).max()
    pa.close()


@pytest.mark.parametrize("hq,hkv,d,requests", [(8, 1, 128, 7), (8, 1, 128, 17), (16, 2, 64, 24), (4, 4, 64, 64), (3, 3, 128, 127), (4, 2, 64, 200)])
@pytest.mark.parametrize("deferred", [False, True])
def test_decode_widely_shared(hq, hkv, d, requests, deferred):
    """Many requests over few chunks: every 16-row group of an item, the last one whole or in part."""
    w = random_case(hq, hkv, d, requests, lens=[700, 40, 129, 64, 1], shared=0)
    _decode(w, range(5), deferred=deferred)
    _decode(w, [0, 3, 4], policy=(64, 8, 1, 1), deferred=deferred)


@pytest.mark.parametrize("hq,hkv,d,requests,chunk", [(32, 8, 128, 15, 192), (32, 8, 128, 16, 64), (32, 8, 128, 32, 192), (16, 8, 64, 65, 320), (8, 8, 128, 127, 128),
                                                     (8, 8, 64, 200, 64), (64, 8, 128, 40, 128)])
@pytest.mark.parametrize("four", ["all", "some"])
def test_decode_many_widely_shared_chunks(hq, hkv, d, requests, chunk, four):
    """Chunks enough for the tcgen05 kernel, 40 per KV head and more: one to several units of 128 query rows each, the last
    one with all its rows, with half of them, or with fewer, which other kernels take; one tile to five, the last one
    ending in its first or its second half."""
    w = random_case(hq, hkv, d, requests, lens=[40 * chunk - 31, 40, 65, 3 * chunk - 1, 1], shared=0)
    _decode(w, range(5) if four == "all" else [0, 3, 4], policy=(chunk, 8, 16, 1), deferred=four == "some")


@pytest.mark.parametrize("hq,hkv,d,requests,chunk", [(32, 8, 128, 32, 192), (8, 8, 64, 200, 64), (32, 8, 128, 3, 256)])
def test_decode_lse_is_exact_to_fp32(hq, hkv, d, requests, chunk):
    """Scores are sums of exact products in fp32.  A score is off by at most (D + 8) 2^-24 of the sum of its products' sizes,
    and by 2^-21 of (sum of q) (lo + 8.5 s), which two fp16 numbers each stand for: with q and k of unit spread 136 * 2^-24 *
    82 * 0.088 + 2^-21 * 4 * 20 * 0.088 = 6e-5, here with a factor of two for larger rows; lse is off by no more."""
    w = random_case(hq, hkv, d, requests, lens=[40 * chunk - 31, 40, 65, 3 * chunk - 1, 1], shared=0)
    _, lse = _decode(w, range(5), policy=(chunk, 8, 16, 1))
    view = View(w, range(5))
    _, ref = OA.decode(view.paths(), view.node_kv, view.q(), hkv)
    assert np.abs(lse - ref).max() <= 1.2e-4


@pytest.mark.parametrize("requests,hkv,copies", [(1, 1, 1), (2, 1, 1), (24, 1, 1), (24, 8, 40)])
def test_decode_scales_far_apart(requests, hkv, copies):
    """Every query row has one token with nearly all of its weight, and values and groups lie up to 2^180 apart: the output
    is that token's value, whatever the tokens before it weighed.  With 40 equal nodes and 8 equal heads there are
    chunks enough for the tcgen05 kernel."""
    d, n, gqa = 128, 200, 8
    rng = np.random.default_rng(13)
    k = rng.choice([-1.0, 1.0], (n, 1, d))
    at = rng.permutation(n)[: requests * gqa].reshape(requests, gqa)
    q = 24 * k[at, 0]
    v = rng.standard_normal((n, 1, 2, d // 2)) * 2.0 ** rng.integers(-90, 91, (n, 1, 2, 1))
    v[:64:2, 0] *= 0.0
    k, q, v = _bf16(k), _bf16(q), _bf16(v.reshape(n, 1, d))
    k, v, q = np.repeat(k, hkv, 1), np.repeat(v, hkv, 1), np.tile(q, (1, hkv, 1))
    path = list(range(copies))
    w = private_workload([n] * copies, [path] * requests, gqa * hkv, hkv, d)
    pa = _handle(w, path)
    for node in path:
        pa.write_node(node, 0, _tensor(k), _tensor(v))
    pa.build()
    out = pa.decode(0, _tensor(q)).double().cpu().numpy()
    kv = kv4.values(k), kv4.values(v)
    ref, _ = OA.decode([path] * requests, lambda _: kv, q, hkv)
    assert pa.status() == 0
    # scores are 24 * 128 * 0.94 / sqrt(128) for a row's token and within 24 * 5 for the others (five standard deviations):
    # the rest weighs less than 2^-190 of it, times 2^180.  Left are the output's rounding (2^-8) and that of p s f to fp16
    # (2^-11 of a term of up to 15 steps s; the group's values spread over 15 steps, at most twice the largest).
    # Where the row's token is 0 the reference is what the rest adds: scores 246 below in log2 give weights that fp32 does
    # not hold, which come out as 0: 200 tokens of 2^-246 times values below 2^93 are below 2^-140
    out, ref = (x.reshape(requests, hkv * gqa, 2, d // 2) for x in (out, ref))
    assert np.all(np.abs(out - ref) <= (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -16) * np.abs(ref).max(-1, keepdims=True) + 2.0 ** -140)
    pa.close()


@pytest.mark.parametrize("requests,hkv,copies", [(1, 1, 1), (24, 1, 1), (24, 8, 40)])
def test_decode_an_outlying_key_that_carries_nothing(requests, hkv, copies):
    """One token's key is 2^30 times the others' and points away from every query: its weight is 0, and the tokens beside it
    in its block and its tile keep theirs."""
    d, n, gqa = 128, 150, 8
    rng = np.random.default_rng(17)
    k, v, q = rng.standard_normal((n, 1, d)), rng.standard_normal((n, 1, d)) / 4, np.abs(rng.standard_normal((requests, gqa, d)))
    k[[7, 100]] = -(2.0 ** 30) * (1 + np.abs(k[[7, 100]]))
    k, v, q = (_bf16(np.repeat(x, hkv, 1)) for x in (k, v, q))
    path = list(range(copies))
    pa = _handle(private_workload([n] * copies, [path] * requests, gqa * hkv, hkv, d), path)
    for node in path:
        pa.write_node(node, 0, _tensor(k), _tensor(v))
    pa.build()
    out = pa.decode(0, _tensor(q)).double().cpu().numpy()
    kv = kv4.values(k), kv4.values(v)
    ref, _ = OA.decode([path] * requests, lambda _: kv, q, hkv)
    assert pa.status() == 0
    assert_close(out, ref, "out")
    pa.close()


@pytest.mark.parametrize("requests,hkv,copies", [(1, 1, 1), (24, 1, 1), (24, 8, 40)])
@pytest.mark.parametrize("gap,large", [(7, 0), (9, 1), (20, 1), (30, 0), (60, 1)])
def test_decode_a_token_whose_groups_lie_far_apart(requests, hkv, copies, gap, large):
    """Keys whose one group of 64 entries is 2^gap times the other, in which the queries are 0, in some blocks of 16 tokens and in
    whole tiles: the scores are those of the other group, to the bound of test_decode_lse_is_exact_to_fp32."""
    d, n, gqa = 128, 200, 8
    rng = np.random.default_rng(23)
    k, v, q = rng.standard_normal((n, 1, 2, 64)), rng.standard_normal((n, 1, d)) / 4, rng.standard_normal((requests, gqa, 2, 64))
    far = np.r_[69, 100:103, 128:200]
    k[far, :, large] *= 2.0 ** gap
    q[:, :, large] = 0.0
    k, v, q = (_bf16(np.repeat(x, hkv, 1)) for x in (k.reshape(n, 1, d), v, q.reshape(requests, gqa, d)))
    path = list(range(copies))
    pa = _handle(private_workload([n] * copies, [path] * requests, gqa * hkv, hkv, d), path)
    for node in path:
        pa.write_node(node, 0, _tensor(k), _tensor(v))
    pa.build()
    lse = torch.empty(requests, gqa * hkv, device="cuda")
    out = pa.decode(0, _tensor(q), lse=lse).double().cpu().numpy()
    kv = kv4.values(k), kv4.values(v)
    ref, ref_lse = OA.decode([path] * requests, lambda _: kv, q, hkv)
    assert pa.status() == 0
    assert np.abs(lse.double().cpu().numpy() - ref_lse).max() <= 1.2e-4
    assert_close(out, ref, "out")
    pa.close()


@pytest.mark.parametrize("requests,hkv,copies", [(1, 1, 1), (24, 1, 1), (24, 8, 40)])
@pytest.mark.parametrize("gap", [-16, -6, 6, 16])
def test_decode_queries_whose_groups_lie_apart_as_the_keys_do_the_other_way(requests, hkv, copies, gap):
    """Both groups of 64 entries add scores of one size.  A query's entries are held to 2^-39 of its row's largest and a group's sum
    of them to 2^-33: times keys 2^16 as large that is below 2^-16 of a score's terms, within the bound of
    test_decode_lse_is_exact_to_fp32."""
    d, n, gqa = 128, 150, 8
    rng = np.random.default_rng(29)
    k, v, q = rng.standard_normal((n, 1, 2, 64)), rng.standard_normal((n, 1, d)) / 4, rng.standard_normal((requests, gqa, 2, 64))
    k[:, :, 1] *= 2.0 ** gap
    q[:, :, 1] *= 2.0 ** -gap
    k, v, q = (_bf16(np.repeat(x, hkv, 1)) for x in (k.reshape(n, 1, d), v, q.reshape(requests, gqa, d)))
    path = list(range(copies))
    pa = _handle(private_workload([n] * copies, [path] * requests, gqa * hkv, hkv, d), path)
    for node in path:
        pa.write_node(node, 0, _tensor(k), _tensor(v))
    pa.build()
    lse = torch.empty(requests, gqa * hkv, device="cuda")
    out = pa.decode(0, _tensor(q), lse=lse).double().cpu().numpy()
    kv = kv4.values(k), kv4.values(v)
    ref, ref_lse = OA.decode([path] * requests, lambda _: kv, q, hkv)
    assert pa.status() == 0
    assert np.abs(lse.double().cpu().numpy() - ref_lse).max() <= 1.2e-4
    assert_close(out, ref, "out")
    pa.close()


def test_a_node_behind_four_gigabytes_of_the_pool():
    """Every kernel that addresses the 4-bit pool, at byte offsets that 32 bits do not hold: write, read, decode, weights and
    eviction of a short node behind one of 60 million tokens."""
    n, far = 200, 60_000_000
    w = private_workload([far, n, 90], [[1], [1]], 2, 1, 64)
    pa = _handle(w, [0, 1, 2], extra_kv4_tiles=far // 64 + 4)   # (only nodes on paths are counted)
    zeros = torch.zeros(far, 1, 64, dtype=torch.bfloat16, device="cuda")
    pa.write_node(0, 0, zeros, zeros)
    del zeros
    k, v = (W.bf16_bits_to_f64(x) for x in w.node_kv_bits(0, 1))
    pa.write_node(1, 0, _tensor(k), _tensor(v))
    from paper_2605_22566_b200 import binding as B
    assert (pa.node_slot(1) - B.gf_pool_info(pa.g).capacity_tiles * 64) // 64 * 4608 > 2 ** 32
    kv = kv4.values(k), kv4.values(v)
    for got, want in zip(pa.load_node(1, 0), kv):
        assert np.array_equal(_bits(got), f64_to_bf16_rne(want))
    pa.build()
    q, lse = pa.make_q(0, "host"), torch.empty(2, 2, device="cuda")
    out = pa.decode(0, q, lse=lse)
    qd = W.bf16_bits_to_f64(w.q_bits(0))
    ref, ref_lse = OA.decode([[1], [1]], lambda _: kv, qd, 1)
    assert_close(out.double().cpu().numpy(), ref, "out")
    weights = pa.new_weights()
    pa.attention_weights(0, q, lse, weights)
    got = pa.node_weights(weights, 1)[0, 0].double().cpu().numpy()
    want = np.exp(np.einsum("rhd,td->rht", qd, kv[0][:, 0]) / 8 - ref_lse[..., None]).sum((0, 1))
    assert np.all(np.abs(got - want) <= 2e-3 * want)          # lse of decode is itself within that
    assert float(weights.sum()) == pytest.approx(4, rel=1e-3)
    (kept,) = pa.evict([(2, 1, 90, 4, 4)], weights)
    idx = kept[0, 0].cpu().numpy()
    for got, all_of in zip(pa.load_node(2, 0), pa.load_node(1, 0)):
        assert torch.equal(got, all_of[idx])
    assert pa.status() == 0
    pa.close()


def test_constant_values_and_equal_keys():
    """Equal keys give the mean of V; constant V comes back exactly (its groups are held exactly)."""
    d, n = 64, 77
    rng = np.random.default_rng(12)
    k = np.broadcast_to(_bf16(rng.standard_normal((1, 2, d))), (n, 2, d)).copy()
    v = np.full((n, 2, d), 0.7109375)
    w = private_workload([n], [[0]], 4, 2, d)
    pa = _handle(w, [0])
    pa.write_node(0, 0, _tensor(k), _tensor(v))
    pa.build()
    q = torch.randn(1, 4, d, device="cuda").to(torch.bfloat16)
    assert torch.equal(pa.decode(0, q), torch.full_like(q, 0.7109375))
    pa.close()


def test_mixed_with_residual_nodes_layers_streams_static_and_capture():
    """4-bit nodes beside a node kept as base + residual, two layers; the static entry point, another stream and a replayed
    graph give the same bits as the plain call."""
    from paper_2605_22566_b200 import binding as B
    lens = [200, 90, 64, 90]
    w = private_workload(lens, [[0, 3], [1, 2], [3], [0, 2]], 8, 2, 128, layers=2)
    pa = _handle(w, [0, 2], max_residual_nodes=1)
    pa.write_nodes("host", skip=[3])
    for layer in (0, 1):
        assert B.gf_node_kv_attach_residual(pa.g, 3, layer, 1, None, None, pa.stream) == B.GF_OK   # node 3 = node 1 as it is
    pa.build()
    for layer in (0, 1):
        q = pa.make_q(layer, "host")
        out = pa.decode(layer, q)
        view = View(w, [0, 2], layer)
        ref, _ = OA.decode(view.paths(), lambda v: view.node_kv(1 if v == 3 else v), view.q(), 2)
        assert_close(out.double().cpu().numpy(), ref, f"layer {layer}")
        other = torch.zeros_like(out)
        assert B.gf_path_attention_decode_static(pa.g, pa.tables, layer, q.data_ptr(), other.data_ptr(), None, pa.stream) == B.GF_OK
        assert torch.equal(other, out)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            third = pa.decode(layer, q, out=torch.zeros_like(out))
        side.synchronize()
        assert torch.equal(third, out)
        graph = torch.cuda.CUDAGraph()
        fourth = torch.zeros_like(out)
        with torch.cuda.graph(graph):
            pa.decode(layer, q, out=fourth)
        for _ in range(2):
            fourth.zero_()
            graph.replay()
            assert torch.equal(fourth, out)
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("four", ["all", "some"])
def test_decode_on_two_streams_captured_on_another_stream_and_twice(four):
    """A batch whose kernels run beside each other: the plain call against fp64, then the same bits from a call on another
    stream, from two captured graphs replayed in turn, and from deferred tables (one stream)."""
    w = two_stream_case(layers=2)
    nodes = list(range(25)) if four == "all" else [0] + list(range(1, 25, 2))
    pa = _handle(w, nodes)
    pa.write_nodes("host")
    pa.build()
    q = [pa.make_q(layer, "host") for layer in (0, 1)]
    out = [pa.decode(layer, q[layer]) for layer in (0, 1)]
    view = View(w, nodes)
    ref, _ = OA.decode(view.paths(), view.node_kv, view.q(), 8)
    assert_close(out[0].double().cpu().numpy(), ref, "out")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = pa.decode(0, q[0], out=torch.zeros_like(out[0]))
    side.synchronize()
    assert torch.equal(other, out[0])
    graphs, outs = [], [torch.zeros_like(out[0]) for _ in (0, 1)]
    for layer in (0, 1):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            pa.decode(layer, q[layer], out=outs[layer])
    for _ in range(3):
        for layer in (0, 1):
            outs[layer].zero_()
            graphs[layer].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(outs[layer], out[layer]) for layer in (0, 1))
    pa.build(deferred=True)
    assert torch.equal(pa.decode(0, q[0]), out[0])
    assert pa.status() == 0
    pa.close()


@pytest.mark.parametrize("requests", [2, 70])
def test_a_captured_step_of_deferred_tables_takes_a_node_written_in_4_bits_later(requests):
    """A graph of a deferred build and its decode, captured while no node is held in 4 bits and replayed when one on its paths is."""
    w = private_workload([200, 130, 64], [[0, 1, 2]] * requests, 4, 2, 64)
    pa = _handle(w, [1])
    pa.write_nodes("host", only=[0, 2])
    pa.build()
    q = pa.make_q(0, "host")
    out = torch.zeros_like(q)
    pa.decode(0, q, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.build(deferred=True)
        pa.decode(0, q, out=out)
    view = View(w, [1])
    for nodes in ([0, 2], [0, 1, 2]):
        if 1 in nodes:
            pa.write_nodes("host", only=[1])
        out.zero_()
        graph.replay()
        ref, _ = OA.decode([nodes] * requests, view.node_kv, view.q(), 2)
        assert_close(out.double().cpu().numpy(), ref, str(nodes))
    assert pa.status() == 0
    pa.close()


def test_extend_refuses_paths_through_4_bit_nodes():
    from paper_2605_22566_b200 import binding as B
    w = private_workload([70, 64, 10], [[0, 2], [1, 2]], 4, 2, 64)
    pa = _handle(w, [1])
    pa.write_nodes("host")
    st, t = B.gf_build_path_tables(pa.g, 2, 4, pa.path_ptr.data_ptr(), pa.path_node.data_ptr(), B.GF_MODE_EXTEND, None, pa.stream)
    assert st == B.GF_ERR_INVALID_PATH and B.gf_tables_bad_request(t) == 1
    pa.close()
