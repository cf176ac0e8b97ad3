"""How far what an 8-bit cache holds may be from what was written, on the definition (tests/reference_cache8.py; the kernels are that byte for byte): the bounds
that the header states.  In units of 2^E, normal codes are 2^-6 and more, whose half step is at most 2^-4 of a value, and below lie multiples of 2^-9.

A row that the growth of its scale moves is rounded again if it leaves the normal codes, by 2^-10 of the scale then; scales at least double, and before the first such
move it was within 2^-4 of a value below 2^-6, so that all of it together is at most 2^-10 (2^-k + 1 + 1/2 + ... + 2^-k) = 2^-9 of the last scale."""
import pytest
import torch

import reference_cache8 as ref


def written(steps):
    """(values, scale) of one block's rows, those of steps [n, D] written one step after the other."""
    D = steps[0].shape[1]
    codes, scales = torch.zeros(1, 1, 32, D, dtype=torch.uint8), torch.zeros(1, 1, 1, dtype=torch.uint8)
    at = 0
    for x in steps:
        ref.write(x[None, :, None], codes, scales, [at], [at + len(x)])
        at += len(x)
    return ref.values(codes, scales)[0, 0, :at], ref.scale_of(scales)[0, 0, 0]


def spread(g, n, D=64, least=-30):
    return (torch.randn(n, D, generator=g, dtype=torch.float64) * 2.0 ** torch.randint(least, 8, (n, D), generator=g)).to(torch.bfloat16)


@pytest.mark.parametrize("seed", range(8))
def test_rows_written_once(seed):
    x = spread(torch.Generator().manual_seed(seed), 32)
    got, scale = written([x])
    x = x.double()
    off, size = (got - x).abs(), x.abs()
    assert (off <= torch.maximum(size * 2.0 ** -4, 2.0 ** -10 * scale)).all()
    kept = size >= 2.0 ** -13 * size.max()
    assert (off <= size * 2.0 ** -4)[kept].all() and not kept.all()


def test_no_further_down_than_that():
    """The largest may be hardly more than half of what its scale reaches: of 225 the value 15 * 2^-10, in the middle between 7 and 8 of the least steps and 2^-13.9
    of it, is off by a fifteenth."""
    x = torch.full((1, 64), 225.0, dtype=torch.float64)
    x[0, 1:] = 15 * 2.0 ** -10
    got, scale = written([x])
    off = (got - x).abs()[0, 1:]
    assert scale == 1 and (off == 2.0 ** -10).all() and 2.0 ** -10 > 15 * 2.0 ** -10 * 2.0 ** -4 and 15 * 2.0 ** -10 > 225 * 2.0 ** -14


@pytest.mark.parametrize("seed", range(16))
def test_rows_that_growth_has_moved(seed):
    g = torch.Generator().manual_seed(seed)
    steps = [spread(g, int(torch.randint(1, 5, (1,), generator=g)), least=-16) * 2.0 ** (i * (1 + seed % 4)) for i in range(6)]
    got, scale = written(steps)
    x = torch.cat(steps).double()
    off = (got - x).abs()
    assert (off <= torch.maximum(x.abs() * 2.0 ** -4, 2.0 ** -9 * scale)).all()


def test_growth_takes_more_than_half_a_step():
    x = (2.0 ** -7 * torch.linspace(1, 2, 256, dtype=torch.float64)).view(4, 64)
    first, second = torch.full((1, 64), 448.0, dtype=torch.float64), torch.full((1, 64), 896.0, dtype=torch.float64)
    got, scale = written([torch.cat([first, x]), second])
    off = (got[1:5] - x).abs().max()
    assert scale == 2 and 2.0 ** -10 * scale < off <= 2.0 ** -9 * scale
