"""The ends of a step from their definitions, in 64 bits or whole numbers (include/basq.h), on the CPU."""
import math

import numpy as np
import torch


def weights(Wq, w_scale, w_zero):
    """fp64 [N, K] of canonical codes: (scale * (code - zero), code, scale and zero point of each weight)"""
    Wq, s, z = Wq.cpu(), w_scale.cpu().double(), w_zero.cpu().double()
    N, KB = Wq.shape
    s, z = s.reshape(N, -1), z.reshape(N, -1)
    q = torch.stack([Wq & 15, Wq >> 4], -1).reshape(N, 2 * KB).double()
    G = 2 * KB // s.shape[1]
    s, z = s.repeat_interleave(G, 1), z.repeat_interleave(G, 1)
    return s * (q - z), q, s, z


def product(x, Wq, w_scale, w_zero, bias=None):
    """(Y, what the sums are made of: sum |s| (32 + |z| + q) |x|), fp64 [M, N]"""
    w, q, s, z = weights(Wq, w_scale, w_zero)
    x = x.cpu().double()
    y, made_of = x @ w.t(), x.abs() @ (s.abs() * (32 + q + z.abs())).t()
    if bias is not None:
        y = y + bias.cpu().double()
        made_of = made_of + bias.cpu().double().abs()
    return y, made_of


def lookup(ids, Wq, w_scale, w_zero, scale):
    w = weights(Wq, w_scale, w_zero)[0] * float(np.float32(scale))
    ids = ids.cpu().long()
    there = (ids >= 0) & (ids < w.shape[0])
    return torch.where(there[:, None], w[ids.clamp(0, w.shape[0] - 1)], torch.zeros(()).double())


def sample_row(row, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """(token, ln of its share, kept) of one row of fp64 logits; weights in the extended type, summed as
    multiples of 2^-bits, the products of the sums with u and top_p rounded to fp64."""
    V = row.size
    row = np.where(np.isnan(row), -math.inf, row)
    index = np.flatnonzero(row > -math.inf)
    if index.size == 0:
        return -1, -math.inf, 0
    index = index[np.argsort(-row[index], kind="stable")]
    if not temperature > 0:
        return int(index[0]), 0.0, 1
    z = row[index].astype(np.longdouble)
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(z == z[0], np.longdouble(1), np.exp((z - z[0]) / np.longdouble(temperature)))
    w = np.where(np.isnan(w), 0, w)
    n = w.size
    if top_k > 0:
        n = min(n, top_k)
    bits = min(50, 62 - (V - 1).bit_length())
    steps = np.rint(w * np.longdouble(2.0 ** bits)).astype(np.uint64)
    running = np.cumsum(steps).astype(np.longdouble)              # (64 bits: exact)
    first = n
    if top_p < 1:
        first = min(first, int(np.searchsorted(running, np.float64(top_p) * np.float64(running[n - 1]), side="left")) + 1)
    if min_p > 0:
        first = min(first, int((w >= min(np.longdouble(min_p), 1)).sum()))
    n = max(first, 1)
    total = running[n - 1]
    u = 0.0 if not u > 0 else min(u, 1.0)
    at = int(np.searchsorted(running[:n], np.float64(u) * np.float64(total), side="right"))
    at = min(at, int(np.flatnonzero(steps[:n])[-1]))
    return int(index[at]), float(np.log(w[at] / total * np.longdouble(2.0 ** bits))), n


def extend(books, seqs, new, page_size, q_len, T):
    """A call of basq_kv_extend on books (dict of lists: lengths, table (rows), free (the free pages), columns, capacity), which are updated:
    dict of positions, slots, starts, batch (pages of each sequence), lengths, status."""
    P, rows = page_size, len(books["lengths"])
    failed = {"positions": [-1] * T, "slots": [-1] * T, "starts": [0] * (len(seqs) + 1), "batch": None, "lengths": [0] * len(seqs)}
    most = books["columns"] * P
    for b, (s, n) in enumerate(zip(seqs, new)):
        if not 0 <= s < rows or s in seqs[:b]:
            return dict(failed, status=[1, b])
        have = books["lengths"][s]
        if not 0 <= have <= most or not 0 <= have + n <= most or (q_len and n > q_len):
            return dict(failed, status=[2, b])
    pages = lambda n: -(-n // P)  # noqa: E731
    change = [pages(books["lengths"][s] + n) - pages(books["lengths"][s]) for s, n in zip(seqs, new)]
    back, wanted = -sum(c for c in change if c < 0), sum(c for c in change if c > 0)
    count = len(books["free"])
    if count + back > books["capacity"]:
        return dict(failed, status=[3, count])
    if wanted > count + back:
        return dict(failed, status=[4, wanted - count - back])
    tokens = sum(max(n, 0) for n in new)
    if not q_len and tokens > T:
        return dict(failed, status=[5, tokens - T])
    for s, c in zip(seqs, change):
        if c < 0:
            had = pages(books["lengths"][s])
            books["free"] += books["table"][s][had + c:had]
    positions, slots, starts, batch = [], [], [0], []
    for s, n, c in zip(seqs, new, change):
        have = books["lengths"][s]
        had = pages(have)
        for i in range(c):
            books["table"][s][had + i] = books["free"].pop()
        run = [(t, books["table"][s][t // P] * P + t % P) for t in range(have, have + n)]
        run = [(-1, -1)] * (q_len - len(run)) + run
        positions += [p for p, _ in run]
        slots += [at for _, at in run]
        starts.append(len(positions))
        books["lengths"][s] = have + n
        batch.append(list(books["table"][s][:pages(have + n)]))
    rest = [-1] * (T - len(positions))
    return {"positions": positions + rest, "slots": slots + rest, "starts": starts, "batch": batch,
            "lengths": [books["lengths"][s] for s in seqs], "status": [0, 0]}
