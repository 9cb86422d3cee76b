"""Values that only a few rows hold, in rows of every way that the kernels hold them: codes that lie on a tie in the layer norm's
own quantiser, and attention rows with infinities and NaN in a later wavefront's part."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_17380_amd.inputs as I
from test_gpu_layernorm import host_bf16, inputs, run, same, wanted
from test_gpu_relbias import LOG16, LOG32, case_inputs
from test_gpu_relbias import run as run_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(6, 100), (6, 511), (6, 700), (6, 1023), (6, 2047), (6, 2048), (2100, 2047), (2100, 2048), (6, 5001),
                                       (900, 5001), (4, 9001), (3, 16386)])
@pytest.mark.parametrize("group,dtype", [(32, torch.float32), (64, torch.bfloat16), (128, torch.float32), (256, torch.bfloat16)])
def test_ties_in_the_norms_quantiser(rows, cols, group, dtype):
    # every group's step is a power of two and half of its values lie midway between two codes, several in each vector of four
    print(f"ties {rows}x{cols} group {group} {dtype}", flush=True)
    rng = np.random.default_rng(cols)
    x = rng.integers(-254, 255, (rows, cols)).astype(np.float32) * np.float32(0.5)
    x[:, ::group] = 127.0
    x *= np.exp2(np.arange(rows) % 5 - 2).astype(np.float32)[:, None]
    assert np.array_equal(x, I.bf16_bits_to_f32(host_bf16(x)))  # 8 bits: exact in bf16 as well
    codes, steps = oracle.act8_pack(x, group)
    assert np.array_equal(steps, np.repeat(np.exp2(np.arange(rows) % 5 - 2).astype(np.float32)[:, None], steps.shape[1], 1))
    _, g, b, dy = inputs(rows, cols, torch.float32, seed=11)
    same(run(x, g, b, dy, dtype, torch.bfloat16, group), wanted(x, g, b, dy, torch.bfloat16, group))


@pytest.mark.parametrize("q,k", [(6, 70), (6, 1100), (6, 2500), (1600, 2048), (900, 2500), (6, 9000)])
@pytest.mark.parametrize("starts,bidirectional", [(LOG32, False), (LOG16, True)])
def test_special_scores_in_a_later_part(q, k, starts, bidirectional):
    print(f"special scores {q}x{k} bidirectional={bidirectional}", flush=True)
    scores, table, dprobs = case_inputs(1, 1, q, k, starts, bidirectional)
    scores[0, 0, 0, :] = -np.inf
    scores[0, 0, 1, :] = np.finfo(np.float32).min
    scores[0, 0, 2, :] = -np.inf
    scores[0, 0, 2, k - 3] = np.nan         # in the last wavefront's part
    scores[0, 0, 3, :k - 9] = -np.inf       # all of the earlier parts
    scores[0, 0, 4, k - 2] = np.inf
    dprobs[0, 0, 5, k - 5] = np.nan
    p, ds, dt = run_rows(1, 1, q, k, starts, bidirectional, scores, table, dprobs, scale=1.0, causal=False)
    v, d = I.bf16_bits_to_f32(p)[0, 0], I.bf16_bits_to_f32(ds)[0, 0]
    want = oracle.relbias_fwd(scores, table, starts, bidirectional, causal=False, scale=1.0)
    fine = [i for i in range(q) if i not in (2, 4)]
    assert np.array_equal(p[0, 0, fine], want[0, 0, fine])
    assert not v[0].any() and not d[0].any()
    assert np.isfinite(v[1]).all() and not v[3, :k - 9].any() and v[3, k - 9:].any()
    for row in (2, 4):
        assert np.isnan(v[row]).all() and np.isnan(d[row]).all()
    assert np.isnan(d[5]).all()
    others = [0, 1, 3] + list(range(6, q))
    want_ds, _ = oracle.relbias_bwd(p, dprobs, starts, bidirectional, causal=False, scale=1.0)
    assert np.array_equal(ds[0, 0, others], want_ds[0, 0, others])
    assert np.isnan(dt).any()
