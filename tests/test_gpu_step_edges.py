"""What stands around a step's attention, at the edges of its contract: refused requests, rows that are not there, entries that are no numbers,
the digits that results hold."""
import numpy as np
import pytest
import torch

from kv4_cases import private_workload
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
