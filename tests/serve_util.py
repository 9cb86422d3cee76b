"""Inputs and caches that the tests of the serving operators share: the oracle's cache on the host and the same on the device."""
import numpy as np
import torch

import oracle
import paper_2609_17380_amd.canon as C
import paper_2609_17380_amd.inputs as I


def tables(rot, positions, theta=5e5):
    """cos, sin fp32 [positions, rot / 2] from binary64."""
    angle = np.arange(positions)[:, None] * theta ** (-np.arange(0, rot, 2) / max(rot, 1))
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def permuted_table(batch, table_len, spare=3, seed=0):
    """(pages, table): every sequence's pages in no order, some pages unused."""
    n = batch * table_len + spare
    return n, np.random.default_rng(seed).permutation(n)[:batch * table_len].reshape(batch, table_len).astype(np.int32)


def host_cache(batch, kv, dim, page, keys, seed=0, fill=(77, np.nan), k=None, v=None):
    """A host cache of `batch` sequences of `keys` tokens; slots that hold none have the codes and steps of `fill`."""
    n, table = permuted_table(batch, max(1, -(-keys // page)), seed=seed)
    c = oracle.KVCache(n, page, kv, dim, table, *fill)
    if k is None:
        k = I.normal_f32((batch, keys, kv, dim), seed, 21) * np.float32(1.5)
    if v is None:
        v = I.normal_f32((batch, keys, kv, dim), seed, 22)
    if keys:
        c.append(k, v, [0] * batch, [keys] * batch)
    return c


def device_cache(c: "oracle.KVCache") -> C.KVCache:
    _, page, kv, dim, _, _ = (int(x) for x in c.dims)
    arrays = [torch.from_numpy(a.copy()).cuda() for a in c.arrays()]
    return C.KVCache(page, kv, dim, *arrays, torch.from_numpy(c.table.copy()).cuda())


def kept(c: "oracle.KVCache", b, keys):
    """The values [keys, kv, dim] that a sequence's keys and values stand for, in 64 bits."""
    _, page, _, _, _, _ = (int(x) for x in c.dims)
    j = np.arange(keys)
    p, s = c.table[b, j // page], j % page
    k = c.k_codes[p, :, s].astype(np.float64) * c.k_steps[p, :, s][..., None]
    v = c.v_codes[p, :, s // 16, :, s % 16].astype(np.float64) * c.v_steps[p, :, s][..., None]
    return k, v


def attention_64(c: "oracle.KVCache", q, scale, starts, q_lens, k_lens, causal, window):
    """The formula in 64 bits over what the cache holds; rows that see nothing are 0."""
    B, Q, H, D = q.shape
    kv = int(c.dims[2])
    out = np.zeros(q.shape)
    for b in range(B):
        n = max(int(k_lens[b]), 0)
        k, v = kept(c, b, n)
        for h in range(H):
            g = h // (H // kv)
            z = q[b, :, h].astype(np.float64) @ k[:, g].T * scale
            pos, j = np.arange(Q)[:, None] + int(starts[b]), np.arange(n)
            seen = np.broadcast_to(np.arange(Q)[:, None] < q_lens[b], z.shape).copy()
            if causal:
                seen &= j <= pos
            if window:
                seen &= np.abs(pos - j) < window
            for i in np.nonzero(seen.any(1))[0]:
                e = np.where(seen[i], np.exp(np.where(seen[i], z[i], -np.inf) - z[i][seen[i]].max()), 0.0)
                out[b, i, h] = e @ v[:, g] / e.sum()
    return out


def from_bf16(u):
    return (np.asarray(u).astype(np.uint32) << 16).view(np.float32)
