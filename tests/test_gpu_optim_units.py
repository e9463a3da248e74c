"""Clipping of lists that one kernel takes and whose blocks have more units than warps: a warp's first unit
waits in registers, the others are read again, and both have to cut a tensor in the same places.

A unit is 4 KB of gradient.  On 152 multiprocessors, three blocks of eight warps on each, units are read again
from 3,649 units on, and one kernel takes a list up to 16,384.  Every element is compared, and what
lies beside the tensors.  The tolerances are those of test_gpu_optim.py: norm and factor within NORM and FACTOR of 64
bits, outputs between the roundings of the two ends."""
import random

import pytest

ap = pytest.importorskip("paper_2108_02416_gb300")
torch = pytest.importorskip("torch")

from test_gpu_optim import (BF16, DEV, F16, F32, NORM, TYPES, check_clip, clip, coef, generator, norms,  # noqa: E402
                            outside, views)

LONG = {F32: 4_000_003, BF16: 8_000_005, F16: 8_000_005}             # 3,907 units
LONGEST = {F32: 15_000_001, BF16: 33_000_001, F16: 33_000_001}       # 14,649 and 16,114


def check(lengths, dtype, offset, out, out_offset):
    gen = generator(40 + offset)
    buffer, ts = views(lengths, dtype, offset, gen)
    target, outs = (buffer, ts) if out is None else views(lengths, out, out_offset, gen, fill=5.0)
    before, mask = [t.clone() for t in ts], outside(target, outs)
    edges, source = target[mask].clone(), buffer.clone()
    want = norms(before)[1]
    got = clip(ts, None if out is None else outs, want / 4)
    assert abs(got - want) <= NORM * want
    check_clip(before, outs, coef(want, want / 4))
    assert torch.equal(target[mask], edges)
    if out is not None:
        assert torch.equal(buffer, source)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset", range(9))
def test_in_place(offset, dtype):
    check([LONG[dtype]], dtype, offset, None, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset", range(9))
@pytest.mark.parametrize("behind", [0, 1, 3, 4, 8])
def test_into_another_tensor(behind, offset, dtype):
    check([LONG[dtype]], dtype, offset, dtype, (offset + behind) % 9)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [(F32, BF16), (BF16, F32), (F16, BF16)])
@pytest.mark.parametrize("offsets", [(0, 0), (4, 4), (5, 0), (0, 6), (7, 3)])
def test_into_another_type(offsets, dtype, out):
    check([LONG[dtype]], dtype, offsets[0], out, offsets[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset", [0, 4, 7])
def test_the_longest_list_of_one_kernel(offset, dtype):
    check([LONGEST[dtype]], dtype, offset, None, 0)
    check([LONGEST[dtype]], dtype, offset, dtype, (offset + 4) % 9)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset", [0, 1, 4, 6])
def test_short_tensors_between_long_ones(offset, dtype):
    n = LONG[dtype]
    lengths = [100, n // 2, 3, 0, 1, n // 3 + 5, 2, 1_023, 5, n, 8, 7]
    check(lengths, dtype, offset, None, 0)
    check(lengths, dtype, offset, dtype, (offset + 4) % 8)


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [4, 5, 6, 7])
def test_few_values_behind_any_address(offset):
    check([0, 1, 2, 3, 4, 5, 7, 8, 9, 1_016, 1_017, 1_020, 1_024], F32, offset, None, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("seed", range(6))
def test_a_flat_vector_cut_at_any_coordinate(seed, dtype):
    rng = random.Random(seed)
    total = rng.randrange(*((4_000_000, 16_000_000) if dtype == F32 else (8_000_000, 32_000_000)))
    cuts = sorted({0, total, *(rng.randrange(total) for _ in range(rng.choice([1, 2, 60, 130])))})
    flat = torch.randn(total, device=DEV, generator=generator(seed)).to(dtype)
    before = flat.clone()
    want = norms([before])[1]
    got = clip([flat[i:j] for i, j in zip(cuts, cuts[1:])], None, want / 4)
    assert abs(got - want) <= NORM * want
    check_clip([before], [flat], coef(want, want / 4))
