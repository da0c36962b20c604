"""GPU tests of the drafting step on a 4-bit cache: what becomes of requests whose length is beyond their block table."""
import numpy as np
import pytest
import torch

import paper_2602_01469_amd as pe
from gpu_harness import max_abs, rel_l2
from oracle import peagle_oracle as orc
from peagle_inputs import bf16_bits_to_f64
from test_gpu_block_cache import BlockRun
from test_gpu_draft_scaled import LSE_ABS, REL, ROWS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("columns", [1, 5, 40])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("K,Hq,Hkv", ROWS)
def test_draft_clamps_lengths_to_the_table(K, Hq, Hkv, D, columns):
    """Flagged, and their results are those of a table full of cached tokens; a length of exactly that is not flagged and gives the
    same bits, one token less does not."""
    print(f"case block clamped lengths K={K} Hq={Hq} D={D} columns={columns}", flush=True)
    full = 64 * columns
    r = BlockRun((full,) * 6, K, Hq, Hkv, D, 7000 + columns, spare=0)
    r.lens = [full, full + 1, full + 64, 2**31 - 1, full - 1, 0]
    r.bt[1:5] = r.bt[0].clone()
    r.table[1:5] = r.table[0]
    r.cl.copy_(torch.tensor(r.lens, dtype=torch.int32))
    for x, host in zip((r.q, r.k, r.v), r.host):   # the same queries and new keys for all
        x[1:] = x[:1].clone()
        host[1:] = host[:1]
    o, lse, status = r.run()
    assert status.tolist() == [0, 1, 1, 1, 0, 0]
    r.lens = [full] * 4 + [full - 1, 0]
    for c in range(6):
        k, v = r.context(c)
        ro, rl = orc.draft_decode(*(bf16_bits_to_f64(x[c]) for x in r.host), k, v, r.shape.scale)
        assert rel_l2(o[c], ro) <= REL and max_abs(lse[c], rl) <= LSE_ABS, c
    if pe.peagle_draft_decode_block_scaled_workspace_bytes(r.shape) < 1024:  # (by request: the same work in the same order)
        assert all(np.array_equal(o[c], o[0]) and np.array_equal(lse[c], lse[0]) for c in (1, 2, 3))
    assert not np.array_equal(lse[4], lse[0])
