"""The gradient of the bias by distance, how many bits its sums keep."""
import numpy as np
import pytest
import torch

import operators_reference as ref
import paper_2202_12429_amd as bp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.mark.parametrize("batch,heads,lq,lk,q_start", [(1, 1, 128, 128, 0), (2, 3, 517, 260, 100), (1, 2, 1500, 1100, 0), (3, 5, 777, 1001, 100)])
@pytest.mark.parametrize("two_sided,borders", [(True, [1, 2, 4, 9, 30, 200]), (False, [])])
def test_gradients_of_fp32_are_summed_in_64_bits(batch, heads, lq, lk, q_start, two_sided, borders):
    """One rounding at the end: half a unit, U of the sum.  The additions in 64 bits are off by less than 2^-53 of the sum of magnitudes
    each, of which no value sees more than the number of pairs."""
    rng = np.random.default_rng(lq)
    rp = bp.make_relpos(borders, two_sided)
    g = rng.normal(size=(batch, heads, lq, lk)).astype(np.float32)              # sums that cancel
    rows = ref.bias_grid(np.zeros((bp.relpos_rows(rp), heads)), borders, two_sided, lq, lk, q_start)[1]
    want, size = ref.bias_grad(g, rows, bp.relpos_rows(rp))
    out = torch.empty(bp.relpos_rows(rp), heads, device=DEV)
    ws = torch.empty(bp.bp_relpos_bias_bwd_workspace_bytes(rp, batch, heads, lq, lk), dtype=torch.uint8, device=DEV)
    bp.bp_relpos_bias_bwd(rp, torch.from_numpy(g).to(DEV), q_start, out, ws)
    off = np.abs(out.double().cpu().numpy() - want)
    assert (off <= U * np.abs(want) + 2 * 2.0 ** -53 * batch * lq * lk * size).all()
