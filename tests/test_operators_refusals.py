"""Calls of the operators for sequences of cached rows that are refused on the host, before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2202_12429_amd as bp


@pytest.fixture
def library(monkeypatch):
    """Notes the entry points that are called, and calls none of them."""
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: calls.append((name, args)) or 0

    import paper_2202_12429_amd.binding as binding
    monkeypatch.setattr(binding, "load_library", Library)
    return calls


@pytest.mark.parametrize("shape,expanded", [((1, 2, 3, 4), (5, 2, 3, 4)), ((5, 1, 3, 4), (5, 2, 3, 4)), ((5, 2, 1, 4), (5, 2, 3, 4)),
                                            ((1, 1, 1, 4), (5, 2, 3, 4)), ((5, 2, 3, 1), (5, 2, 3, 4))])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_expanded_arrays_are_not_taken_for_dense_ones(shape, expanded, dtype, library):
    """What autograd gives for a bias that a batch shares has a stride of 0, which the library reads as "dense"."""
    rp, g = bp.make_relpos([1, 2]), torch.ones(shape, dtype=dtype).expand(expanded)
    with pytest.raises(ValueError):
        bp.bp_relpos_bias_bwd(rp, g, 0, torch.zeros(3, 2), torch.zeros(4096, dtype=torch.uint8), stream=0)
    if g[0].stride() != g[0].contiguous().stride():
        with pytest.raises(ValueError):
            bp.bp_relpos_bias_fwd(rp, torch.zeros(3, 2), 0, g[0], stream=0)
    assert not library


def test_strides_of_sizes_of_one_do_not_matter(library):
    """An expanded dimension of size 1 is in memory as it is."""
    rp, g = bp.make_relpos([1, 2]), torch.ones(2, 3, 4)
    for t in (g.expand(1, 2, 3, 4), g[None].as_strided((1, 2, 3, 4), (0, 12, 4, 1)), g[None, :, :1].as_strided((1, 2, 1, 4), (0, 12, 0, 1))):
        bp.bp_relpos_bias_bwd(rp, t, 0, torch.zeros(3, 2), torch.zeros(4096, dtype=torch.uint8), stream=0)
    assert [name for name, _ in library] == ["bp_relpos_bias_bwd"] * 3
    assert all(args[7:10] == want for (_, args), want in zip(library, [(4, 12, 0), (4, 12, 0), (0, 12, 0)]))


def status(call, *args):
    with pytest.raises(bp.BagpipeError) as e:
        call(*args)
    return e.value.status


def test_bias_gradients_of_more_work_than_a_launch_holds():
    rp = bp.make_relpos([1, 2], True)
    size = bp.bp_relpos_bias_bwd_workspace_bytes
    for lq, lk in ((1 << 20, 1), ((1 << 20) - 1, 1), (1 << 18, 3 << 20), (1, (1 << 30) - 1), (1 << 10, (1 << 30) - (1 << 10))):
        assert size(rp, 1, 1, lq, lk) > 0                                   # lq * (lq + lk) up to 2^40
    for lq, lk in ((1 << 21, 1), ((1 << 30) - 1, 1), (1 << 21, 1 << 19)):
        assert status(size, rp, 1, 1, lq, lk) == -6


def test_borders_that_32_bits_do_not_hold():
    for bad in ([1.5, 2.5], np.array([1, (1 << 32) + 5]), [[1, 2], [3, 4]], [float("nan")]):
        with pytest.raises(ValueError):
            bp.make_relpos(bad)
    for good in ([], range(1, 5), (2, 9), np.array([3, 7]), torch.tensor([1, 4]), [1.0, 2.0]):
        assert bp.relpos_rows(bp.make_relpos(good)) == len(good) + 1


def test_strides_whose_span_overflows():
    """A head's span of (lq - 1) * row_stride + lk elements is computed in 64 bits."""
    rp, lib = bp.make_relpos([1]), bp.load_library()
    table, out = torch.zeros(2, 2), torch.zeros(2, 1, 5)
    for lq, row in ((1 << 20, 1 << 44), ((1 << 30) - 1, 1 << 45), (1 << 28, 1 << 36), (2, 1 << 45)):
        assert lib.bp_relpos_bias_fwd(ctypes.byref(rp), table.data_ptr(), 2, lq, 5, 0, out.data_ptr(), 0, row, 5, None) == -1
    assert lib.bp_relpos_bias_fwd(ctypes.byref(rp), table.data_ptr(), 2, 0, 5, 0, out.data_ptr(), 0, 1 << 45, 0, None) == 0


def test_a_cap_too_small_for_its_scale():
    cfg = bp.make_config(100, 100, 64)
    size = lambda **kw: bp.bp_embbag_attn_fwd_workspace_bytes(cfg, bp.make_attn(2, 1, 16, **kw), 10, 2)
    for scale, cap in ((1.0, 1e-39), (1e30, 1e-10), (-1e38, 0.1)):
        assert status(lambda: size(scale=scale, cap=cap)) == -1
    for scale, cap in ((1.0, 1e-38), (0.0, 1e-39), (1e30, 0.0)):
        assert size(scale=scale, cap=cap) >= 0
