"""Scales of int8 rows whose norm's factor is no fp32 number, while the scale is one, against 64 bits: with a large gain over
the smallest rows the factor is above 2^128, with the largest rows below 2^-126.  The scale is max|u| / 127 (two
roundings, 2^-24 each) times a factor in 64 bits, rounded once."""
import numpy as np
import pytest
import torch

from paper_2608_14586_amd import binding as vb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 896, 4096])
@pytest.mark.parametrize("summed", [False, True])
def test_factors_outside_fp32(d, summed):
    rng = np.random.default_rng(d)
    size = np.array([2.0 ** -138, 2.0 ** -130, 2.0 ** -128, 2.0 ** -127, 2.0 ** -110, 2.0 ** 120, 2.0 ** 125, 2.0 ** 126])[:, None]
    x = (rng.uniform(0.5, 1.9, (len(size), d)) * rng.choice([-1, 1], (len(size), d)) * size).astype(np.float32)
    for g in (np.float32(2.0 ** 60), np.float32(0.75)):
        gain = (rng.uniform(0.5, 1.0, d) * g).astype(np.float32)
        rows = x[:5] if g > 1 else x[5:]  # t g in range
        codes, scales = torch.empty(rows.shape, dtype=torch.int8, device="cuda"), torch.empty(len(rows), device="cuda")
        total = torch.empty(rows.shape, device="cuda") if summed else None
        vb.vla_op_norm_i8(torch.from_numpy(rows).cuda(), None, total, torch.from_numpy(gain).cuda(), 0.0, codes, scales)
        u = (rows * gain).astype(np.float64)
        top = np.abs(u).max(1, keepdims=True)
        assert np.isfinite(u).all() and (top > 2.0 ** -100).all()
        assert np.array_equal(codes.cpu().numpy(), np.rint(127 * u / top))
        want = top[:, 0] / 127 / np.sqrt((rows.astype(np.float64) ** 2).mean(1))
        assert np.all(np.abs(scales.cpu().numpy() - want) <= 3 * 2.0 ** -24 * want)
