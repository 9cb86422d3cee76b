"""int8 products of whole 256 x 256 tiles on both sides of the number that the pipelined kernel takes (half of the CUs), with a step for
every row and with one for the tensor, and raw sums: exact."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_17380_amd.canon as C
import paper_2609_17380_amd.inputs as I
from gpu_util import DEV, assert_bits, dev_f32, host_f32, host_u16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(1792, 4096, 64), (2048, 4096, 64), (2304, 4096, 128), (4096, 2816, 192), (256, 32768, 64)])
def test_whole_tiles(m, n, k):
    rng = np.random.default_rng(m)
    a, b = (rng.integers(-128, 128, s).astype(np.int8) for s in ((m, k), (n, k)))
    sa, sb = (np.exp(I.normal_f32((x,), x, 62)).astype(np.float32) for x in (m, n))
    da, db, dsa, dsb = torch.from_numpy(a).to(DEV), torch.from_numpy(b).to(DEV), dev_f32(sa), dev_f32(sb)
    want = oracle.gemm_i8_tokens(a, sa, b, sb)
    for pad in (0, 8):
        y = torch.full((m, n + pad), 7.0, device=DEV)
        C.gemm_i8_tokens(m, n, k, da, k, dsa, db, k, dsb, y, ldc=n + pad)
        h = torch.full((m, n + pad), 7.0, dtype=torch.bfloat16, device=DEV)
        C.gemm_i8_tokens(m, n, k, da, k, dsa, db, k, dsb, h, ldc=n + pad)
        torch.cuda.synchronize()
        assert (y[:, n:] == 7.0).all() and (h[:, n:] == 7.0).all()
        assert_bits(host_f32(y[:, :n].contiguous()), want, "fp32")
        assert_bits(host_u16(h[:, :n].contiguous()), torch.from_numpy(want).bfloat16().view(torch.int16).numpy().view(np.uint16),
                    "bf16")
    one = sa[:1].copy()
    want = oracle.gemm_i8_tokens(a, np.repeat(one, m), b, sb)
    y, acc = torch.empty(m, n, device=DEV), torch.empty(m, n, dtype=torch.int32, device=DEV)
    C.gemm_i8(m, n, k, da, k, db, k, acc=acc, y=y, sa=dev_f32(one), sb=dsb)
    torch.cuda.synchronize()
    assert_bits(host_f32(y), want, "tensor's step")
    assert (acc.cpu().numpy() == (a.astype(np.float32) @ b.astype(np.float32).T).astype(np.int32)).all()  # sums below 2^24: exact
