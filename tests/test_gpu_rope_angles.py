"""The angle's part of a rotation's error (needs a gfx950 GPU).

A pair (1, 0) turns into cosine and sine themselves.  In fp32 the angle in half turns,
up to 1, would be off by 2^-25 of one (pi 2^-25 rad); its remainder goes in by the
first order, so that the functions' own error is what is left: at most 4 steps, as
OpenCL asks of sinpi and cospi, and half a step of the multiply-add.  A step is at
most 2^-23 of the value.  Near the zeros of either function that is far below the
angle's error."""
from __future__ import annotations

import pytest
import torch

from paper_2606_00024_amd import _lib, api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    _lib.load()
    yield


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("far", [4096, 131072])
def test_cosines_and_sines_are_those_of_64_bits(far, layout):
    rows = 8192
    gen = torch.Generator().manual_seed(far)
    positions = torch.randint(0, far, (rows,), generator=gen).int()
    freqs = 10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)
    first, second = (slice(0, 64), slice(64, 128)) if layout == "half" else (slice(0, 128, 2), slice(1, 128, 2))
    x = torch.zeros(rows, 1, 128)
    x[..., first] = 1.0
    got = api.rope_rows(x.to(DEV), positions.to(DEV), api.Rope(freqs.to(DEV), layout)).cpu().double()[:, 0]
    angle = positions.double()[:, None] * freqs
    for value, want in ((got[:, first], angle.cos()), (got[:, second], angle.sin())):
        # 64 bits: the angle's own product and the reduction, 2^-51 of the angle
        bound = 4.5 * 2.0 ** -23 * want.abs() + 2.0 ** -51 * angle + 2.0 ** -44
        assert bool(((value - want).abs() <= bound).all())
        assert int((want.abs() < 0.05).sum()) > 1000          # where the angle would show
