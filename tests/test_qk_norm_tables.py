"""Rotary arguments of qk_norm_rotate that leave part of the others out are refused: rows asked to be rotated do not come back as they
were (no GPU needed)."""

import pytest
import torch


@pytest.mark.parametrize("given", [("sin",), ("positions",), ("sin", "positions"), ("cos",), ("cos", "sin"), ("cos", "positions")])
def test_part_of_them(given):
    import paper_2607_28699_gb300 as wc
    x = torch.zeros(5, 6, 128, dtype=torch.float16)
    every = dict(positions=torch.zeros(5, dtype=torch.int32), cos=torch.zeros(8, 64), sin=torch.zeros(8, 64))
    with pytest.raises(ValueError):
        wc.qk_norm_rotate(x[:, :4], x[:, 4:], **{n: every[n] for n in given}, stream=torch.Stream("cpu"))
