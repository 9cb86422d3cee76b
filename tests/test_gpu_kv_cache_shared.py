"""canon_cache_append where sequences share pages: different slots of one 16-token group from several sequences, the same token to one
slot, and two tokens to one slot, which leaves every other slot as it should be."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_17380_amd.canon as C
import paper_2609_17380_amd.inputs as I
from gpu_util import dev_f32, dev_i32
from serve_util import device_cache

pytestmark = pytest.mark.gpu


def shared(B, KV, D, page, pages):
    """A cache whose sequences all have the same pages."""
    n = pages + 2
    order = np.random.default_rng(D).permutation(n)[:pages].astype(np.int32)
    return oracle.KVCache(n, page, KV, D, np.repeat(order[None], B, 0), 55, np.nan)


def append(cache, c, k, v, starts, lens):
    B, Q, KV, D = k.shape
    C.cache_append(cache, C.CacheRows(B, Q, q_starts=dev_i32(np.asarray(starts)), q_lens=dev_i32(np.asarray(lens))),
                   dev_f32(k).view(B * Q, KV * D), dev_f32(v).view(B * Q, KV * D))
    c.append(k, v, starts, lens)
    torch.cuda.synchronize()


def differing(cache, c):
    """[n_pages, heads, page]: slots that are not the oracle's."""
    kc, vc, ks, vs = (t.cpu().numpy() for t in cache.tensors)
    n, page = ks.shape[0], ks.shape[2]
    per_slot = lambda x: x.transpose(0, 1, 2, 4, 3).reshape(n, x.shape[1], page, -1)  # noqa: E731
    steps = lambda a, b: a.view(np.uint32) != b.view(np.uint32)  # noqa: E731
    return ((kc != c.k_codes).any(-1) | (per_slot(vc) != per_slot(c.v_codes)).any(-1) | steps(ks, c.k_steps) | steps(vs, c.v_steps))


def tokens(B, Q, KV, D, seed):
    return (I.normal_f32((B, Q, KV, D), seed, s) * np.float32(2) for s in (101, 102))


@pytest.mark.parametrize("D,KV,page", [(32, 2, 16), (96, 1, 32), (128, 4, 64), (256, 2, 256)])
def test_different_slots(D, KV, page):
    B, Q = 24, 5
    c = shared(B, KV, D, page, -(-(B * Q + 3) // page))
    cache = device_cache(c)
    k, v = tokens(B, Q, KV, D, 1)
    append(cache, c, k, v, 3 + Q * np.arange(B), [Q] * B)  # one run of positions, five of each sequence
    assert not differing(cache, c).any()
    k, v = tokens(B, 1, KV, D, 2)
    append(cache, c, k, v, 2 * np.arange(B), [1] * B)
    assert not differing(cache, c).any()


def test_one_slot():
    B, KV, D, page = 8, 2, 64, 16
    c = shared(B, KV, D, page, 3)
    cache = device_cache(c)
    k, v = tokens(B, 40, KV, D, 3)
    append(cache, c, np.repeat(k[:1], B, 0), np.repeat(v[:1], B, 0), [2] * B, [40] * B)  # the same tokens of every sequence
    assert not differing(cache, c).any()
    append(cache, c, k, v, [2] * B, [1, 20, 20, 20, 20, 7, 0, 1])  # positions 2 .. 21 twice and more
    bad = differing(cache, c)
    twice = np.zeros_like(bad)
    pos = np.arange(2, 22)
    twice[c.table[0, pos // page], :, pos % page] = True
    assert not (bad & ~twice).any()
