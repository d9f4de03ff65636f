"""Inputs that show how many digits a projection's results hold, what they may be off by, and, on the host, what coarser arithmetic would be off by."""
import numpy as np
import torch

MMA_K, CHUNK_K = 16, 512     # entries of K in one addition of the tensor cores; in the sums that they add up by themselves where results are fp32


def same_sign(rows, k, n, seed=0):
    """x [rows, k] and w [n, k] in bf16, all positive, so that every addition that is cut off makes a sum smaller."""
    gen = torch.Generator().manual_seed(seed)
    return (torch.rand(rows, k, generator=gen) + 0.5).to(torch.bfloat16), (torch.rand(n, k, generator=gen) + 0.5).to(torch.bfloat16)


# A cut off addition takes half a unit in the last place in the mean, at most 2^-24 of the sum so far.  32 additions (512 entries of K), the sum growing evenly:
# 16.5 of those, 9.8e-7; the sums of 512 entries are added with rounding, at most 2^-25 in the mean and either way: 64 of them are off by 2^-22, 2.4e-7, if no two errors cancel.
SAME_SIGN = 16.5 * 2.0 ** -24 + 2.0 ** -22


def cut(x):
    """fp64 values cut off (not rounded) to fp32."""
    y = x.astype(np.float32)
    return np.where(np.abs(y.astype(np.float64)) > np.abs(x), np.nextafter(y, np.float32(0)), y).astype(np.float64)


def sums_cut_off(x, w, chunk):
    """x w^T with every addition of 16 products cut off, sums taken out and added with rounding every `chunk` entries of K."""
    x, w = x.double().numpy(), w.double().numpy()
    total = np.zeros((x.shape[0], w.shape[0]))
    for c in range(0, x.shape[1], chunk):
        acc = np.zeros_like(total)
        for k in range(c, min(c + chunk, x.shape[1]), MMA_K):
            acc = cut(acc + x[:, k:k + MMA_K] @ w[:, k:k + MMA_K].T)
        total = (total + acc).astype(np.float32).astype(np.float64)
    return total


LEADING, REST = 1 + 2.0 ** -10 * (2 - 2.0 ** -7), 2.0 ** -18 - 2.0 ** -21


def between_numbers(rows, n, adapters, rank):
    """x, a, b in bf16: every entry of h = A x is an fp32 number, the row's power of two times LEADING + REST, of which two bf16 numbers hold LEADING, less nearly half a step of
    the second and always to the same side; b is positive."""
    x = torch.zeros(rows, 16)
    x[:, :8] = (2.0 ** (torch.arange(rows) % 5 - 2.0)).unsqueeze(1)
    a = torch.zeros(adapters, rank, 16)
    a[:, :, 0], a[:, :, 1], a[:, :, 2] = 1.0, LEADING - 1, REST
    gen = torch.Generator().manual_seed(n)
    b = torch.rand(adapters, n, rank, generator=gen) + 0.5
    return tuple(t.to(torch.bfloat16) for t in (x, a, b))


def cancelling(x, b):
    """w [n, in] in bf16 so that w x takes LEADING of between_numbers' b h away: what is left of their sum is REST."""
    left = -LEADING * b.double().sum(1)
    w = torch.zeros(b.shape[0], x.shape[1], dtype=torch.bfloat16)
    for i in range(8):
        w[:, i] = left.to(torch.bfloat16)
        left = left - w[:, i].double()
    assert not left.any()
    return w


# Three bf16 numbers hold 24 bits: these h exactly.  What is left is the additions of the three products, 16 ranks at a time (64 ranks: 12 additions), and two more that join them
# to the rest, each cut off by at most 2^-23.
THREE = 14 * 2.0 ** -23
# Two: half a step of the second, which is below 2^-9 of these values, and 10 additions.
TWO = 2.0 ** -18 + 10 * 2.0 ** -23


def in_numbers(h, numbers):
    """h in that many bf16 numbers, each the nearest to what is left."""
    left, total = h.double(), torch.zeros_like(h, dtype=torch.float64)
    for _ in range(numbers):
        part = left.to(torch.float32).to(torch.bfloat16).double()
        total += part
        left = left - part
    return total
