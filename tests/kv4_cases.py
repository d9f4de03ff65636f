"""Workloads over nodes held in 4 bits, in bf16, or some each, and the oracle's view of them."""
import numpy as np

from oracle import kv4
from paper_2605_22566_b200 import workloads as W


def private_workload(lens, paths, hq, hkv, d, layers=1, seed=5, **over):
    """Every node a request's own (no edges)."""
    return W.Workload(name="kv4", config_id=-1, seed=seed, mode="decode", num_layers=layers, num_q_heads=hq, num_kv_heads=hkv, head_dim=d,
                      num_shared_nodes=0, num_nodes=len(lens), edge_src=np.zeros(0, np.int32), edge_dst=np.zeros(0, np.int32),
                      node_len=np.array(lens, np.int32), path_ptr=np.concatenate([[0], np.cumsum([len(p) for p in paths])]).astype(np.int32),
                      path_node=np.array(sum(paths, []), np.int32), **over)


class View:
    """fp64 states of a workload's nodes (the values that the codes stand for, where held in 4 bits) and its queries."""

    def __init__(self, w, four, layer=0):
        self.w, self.four, self.layer, self.cache = w, set(four), layer, {}

    def node_kv(self, v):
        if v not in self.cache:
            k, vv = (W.bf16_bits_to_f64(x) for x in self.w.node_kv_bits(self.layer, v))
            self.cache[v] = (kv4.values(k), kv4.values(vv)) if v in self.four else (k, vv)
        return self.cache[v]

    def q(self):
        return W.bf16_bits_to_f64(self.w.q_bits(self.layer))

    def paths(self):
        return [[v for v in self.w.path(r).tolist() if self.w.node_len[v] > 0] for r in range(self.w.num_requests)]


#: node lengths that end inside a tile, a block of 16 tokens, or neither; 0 among them
ODD_LENS = [1, 15, 16, 17, 63, 64, 65, 0, 130, 257]


def random_case(hq, hkv, d, requests, lens=ODD_LENS, seed=3, shared=None, **over):
    """`requests` paths over random subsets of the nodes; node `shared`, if given, is on every path."""
    rng = np.random.default_rng(seed)
    paths = []
    for _ in range(requests):
        p = rng.permutation(len(lens))[:rng.integers(1, 5)].tolist()
        if shared is not None:
            p = [shared] + [v for v in p if v != shared]
        paths.append(p)
    return private_workload(lens, paths, hq, hkv, d, seed=seed, **over)


def two_stream_case(hq=32, hkv=8, d=128, layers=1):
    """Enough of widely shared and of unshared chunks that a call runs its kernels on two streams: 40 requests over one long
    node, 24 of them over a node of their own as well."""
    return private_workload([5000] + [300] * 24, [[0] + ([1 + r] if r < 24 else []) for r in range(40)], hq, hkv, d, layers=layers)
