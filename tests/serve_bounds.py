"""How far attention over a cache in 8 bits may be from the formula: a bound for every element, of what the row itself adds up."""
import numpy as np

import paper_2609_17380_amd.inputs as I
from serve_util import from_bf16, host_cache, kept


def attention_bound(c, q, scale, starts, q_lens, k_lens, causal=True, window=0):
    """(formula in 64 bits, bound), both [batch, q_len, heads, dim], of what R26 may differ by.  With w_j the weights (of sum 1)
    of a row's keys, M = sum w_j |v_j| for each element and T = sum w_j max |v_j| over the head:
      output    rounded to bf16: 2^-8 |o|
      weights   each off by a part dz of itself where its score is off by dz: 2 dz M in all.  dz: a query element by half of 2^s,
                2^s <= 2^-21 of the query's largest, unless it is a multiple of that (bf16 down to 2^-14 of the largest), times
                scale |k|; the roundings on the way to a score's exponent, at most 8 of 2^-24 of |z|; the exponential 1.6e-7
      products  of weight and value step to half a multiple of 2^s, 2^s <= 2^-21 of a tile's largest: 256 keys by 2^-22 each of the
                largest w_j max |v_j| (a token's largest code is 127), below 2^-14 of the tile's part of T; never less than
                half of 2^-126 on 256 codes of 127: 2^-112 a tile, of a sum of weights of at least 1/2 (most steps are half as
                large as these bounds take them)
      sums      in binary32: 64 roundings of a tile's chain, tree and conversions and 4 a tile, of M
    A weight below 2^-126 of its tile's reference is left out: keys times that of the largest value."""
    B, Q, H, D = q.shape
    kv = int(c.dims[2])
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        n = max(int(k_lens[b]), 0)
        k, v = kept(c, b, n)
        tiles = -(-n // 256)
        for h in range(H):
            g = h // (H // kv)
            z = q[b, :, h].astype(np.float64) @ k[:, g].T * scale
            pos, j = np.arange(Q)[:, None] + int(starts[b]), np.arange(n)
            seen = np.broadcast_to(np.arange(Q)[:, None] < q_lens[b], z.shape).copy()
            if causal:
                seen &= j <= pos
            if window:
                seen &= np.abs(pos - j) < window
            av = np.abs(v[:, g])
            for i in np.nonzero(seen.any(1))[0]:
                w = np.where(seen[i], np.exp(np.where(seen[i], z[i], -np.inf) - z[i][seen[i]].max()), 0.0)
                w /= w.sum()
                o, M, T = w @ v[:, g], w @ av, w @ av.max(-1)
                step = 2.0 ** (np.frexp(np.abs(q[b, i, h]).max())[1] - 22)
                off = np.where(np.float64(q[b, i, h]) % step == 0, 0.0, step / 2)
                dz = (np.abs(k[:, g]) @ off)[seen[i]].max() * abs(scale) + 8 * 2.0 ** -24 * np.abs(z[i][seen[i]]).max() + 1.6e-7
                out[b, i, h] = o
                bound[b, i, h] = (2.0 ** -8 * np.abs(o) + (2.1 * dz + (64 + 4 * tiles) * 2.0 ** -24) * M + 2.0 ** -14 * T +
                                  tiles * 2.0 ** -111 + n * 2.0 ** -126 * av.max(initial=0.0))
    return out, bound


def spread_case(kind, size, B=1, KV=2, G=2, D=64, K=1024, Q=3, page=16):
    """(cache, queries): tokens whose values are of very different sizes.  "none": one token of every 256 has values `size` times
    the others' and a score 40 below them.  "some": sizes spread by e^(size normal), peaked weights.  "all": all alike."""
    H = KV * G
    q = I.normal_f32((B, Q, H, D), 3, 81)
    k, v = (I.normal_f32((B, K, KV, D), 3, s) for s in (82, 83))
    if kind == "none":
        q[..., 0], k[..., 0] = 8.0, 0.0
        for j in range(97, K, 256):
            k[:, j] = 0.0
            k[:, j, :, 0] = -40.0  # times 8 and the scale 1/8
            v[:, j] *= np.float32(size)
    elif kind == "some":
        q *= np.float32(3)
        v *= np.exp(size * I.normal_f32((B, K, KV, 1), 3, 84)).astype(np.float32)
    else:
        v *= np.float32(size)
    return host_cache(B, KV, D, page, K, k=k, v=v), q


SPREADS = [("none", 1e2), ("none", 1e3), ("none", 1e5), ("none", 1e9), ("some", 2.0), ("some", 6.0), ("all", 1e-30), ("all", 1e30)]


def outlier_case(times, bf16=False, B=1, KV=2, G=2, D=64, K=700, Q=3, page=16):
    """(cache, queries): one channel of every query `times` the others, and keys with as much less in it."""
    q = I.normal_f32((B, Q, KV * G, D), 5, 91)
    k, v = (I.normal_f32((B, K, KV, D), 5, s) for s in (92, 93))
    q[..., 7] = times * (1 + np.abs(q[..., 7]))
    k[..., 7] /= np.float32(times)
    k[:, ::50, :, 7] = 1.0 / 127.0  # and here and there a code's worth of it
    if bf16:
        q = from_bf16(q.view(np.uint32) >> 16)
    return host_cache(B, KV, D, page, K, k=k, v=v), q


OUTLIERS = [(30.0, False), (1e3, False), (1e4, False), (30.0, True), (1e3, True), (1e4, True)]
