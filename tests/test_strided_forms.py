"""Column forms that are strided views: what the binding brings into rows, and what it leaves to be refused.  CPU only."""
import pytest
import torch

import paper_2608_16157_amd as ftm


def form(rows=256, cols=100):
    c = ftm.ActCodes(rows, cols, device="cpu")
    c.codes.copy_(torch.arange(rows * 128).view(rows, 128) % 251)
    c.scales.copy_(torch.arange(256).view(1, 256))
    return c


def test_views_are_brought_into_rows():
    c = form()
    turned = ftm.ActCodes.of(c.codes.t().contiguous().t(), c.scales, 256, 100)
    got = ftm._laid_out(turned, None)
    assert got.codes.is_contiguous() and torch.equal(got.codes, c.codes) and got.scales is c.scales
    assert (got.rows, got.cols) == (256, 100) and not turned.codes.is_contiguous()
    wide = torch.zeros(2, 300, dtype=torch.uint8)
    wide[1:, 20:276] = c.scales
    got = ftm._laid_out(ftm.ActCodes.of(c.codes, wide[1:, 20:276].expand(1, 256)[:, ::1], 256, 100), None)
    assert torch.equal(got.scales, c.scales) and got.codes is c.codes


def test_what_is_in_rows_or_fits_no_form_goes_on_as_it_is():
    c = form()
    assert ftm._laid_out(c, None) is c
    for bad in (None, 3, ftm.ActCodes.of(c.codes.t(), c.scales, 256, 100), ftm.ActCodes.of(c.codes[:, ::2], c.scales, 256, 100),
                ftm.ActCodes.of(None, c.scales, 256, 100)):
        assert ftm._laid_out(bad, None) is bad


def test_forms_off_the_device_are_refused_all_the_same():
    turned = ftm.ActCodes.of(torch.zeros(256, 256, dtype=torch.uint8).t(), torch.zeros(2, 256, dtype=torch.uint8), 256, 256)
    with pytest.raises(ValueError, match="device"):
        ftm.ft_linear_weight_grad(256, 256, 256, turned, turned, torch.zeros(256, 256))
