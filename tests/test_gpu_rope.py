"""Rotary positions of part of a head on the GPU against the float64 oracle.

Tolerance: fp32 arithmetic on the fp32 table (three roundings of terms of size
|a cos| + |b sin|), then one rounding to the output type with unit roundoff u
(bf16 2^-8, fp16 2^-11 and half a subnormal step 2^-25, fp32 2^-24)."""

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2605_30351_gb300 import videomla as V

pytestmark = pytest.mark.gpu

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    V.load()
    V.mla_device_status(clear=True)
    yield
    assert V.mla_device_status(clear=True) == V.MLA_OK


def make(pairs, length=300, offset=0, half=False, axes=None, scaling=0, factor=1.0):
    tab = V.mla_rope_scaled_table_fill(2 * sum(pairs), length, scaling=scaling, factor=factor,
                                       native_len=64)
    return tab, V.Rope(torch.from_numpy(tab).cuda(), pairs, offset=offset, half=half, axes=axes)


def draw(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def check(x, y, tab, rope, pos, half, offset, inverse=False, keep=None):
    xs, ys = x.double().numpy(), y.double().cpu().numpy()
    ref = O.rotate(xs, pos.numpy(), tab, rope.pairs, offset, half, inverse)
    u = UNIT[x.dtype]
    size = O.rotate(np.abs(xs), pos.numpy() * 0, np.broadcast_to(
        np.abs(tab).max() * np.array([1.0, 1.0]), tab.shape), rope.pairs, offset, half, False)
    bound = u * np.abs(ref) + 2.0 ** -22 * (np.abs(xs) + np.abs(size)) + 2.0 ** -25
    assert (np.abs(ys - ref) <= bound).all(), np.max(np.abs(ys - ref) / bound)
    m2 = 2 * sum(rope.pairs)
    same = np.ones(xs.shape[2], bool)
    same[offset:offset + m2] = False
    assert np.array_equal(ys[:, :, same], xs[:, :, same])


CASES = [
    # tokens, heads, dim, pairs, offset, half
    (1, 1, 32, (6, 5, 5), 0, False),
    (7, 12, 32, (6, 5, 5), 0, False),
    (33, 12, 128, (6, 5, 5), 96, False),
    (33, 12, 128, (32, 0, 0), 0, True),
    (5, 3, 96, (16, 0, 0), 64, True),
    (9, 5, 80, (24, 0, 0), 16, True),
    (4, 2, 24, (3, 2, 1), 6, False),        # offset and width off the 16-byte grid
    (4, 2, 25, (3, 2, 1), 7, True),         # odd head width and offset
    (3, 40, 256, (128, 0, 0), 0, True),     # more items than a block has threads
    (257, 1, 64, (32, 0, 0), 0, False),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("inverse", [False, True])
def test_matches_oracle(case, dtype, inverse):
    tokens, heads, dim, pairs, offset, half = CASES[case]
    tab, rope = make(pairs, offset=offset, half=half, scaling=3 if case % 2 else 0,
                     factor=4.0 if case % 2 else 1.0)
    x = draw((tokens, heads, dim), dtype, case)
    pos = torch.randint(0, 300, (tokens, rope.axes), dtype=torch.int32,
                        generator=torch.Generator().manual_seed(case))
    y = torch.full_like(x, float("nan"), device="cuda")
    V.mla_rope_apply(rope, x.cuda(), pos.cuda(), y, inverse=inverse)
    check(x, y, tab, rope, pos, half, offset, inverse)
    z = x.cuda()                                      # in place
    V.mla_rope_apply(rope, z, pos.cuda(), z, inverse=inverse)
    assert torch.equal(z, y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("lead,tail", [(0, 0), (1, 0), (8, 3)])
def test_strides_and_alignment(dtype, half, lead, tail):
    """Views into larger tensors (heads first, odd starts), neighbours intact."""
    tokens, heads, dim = 13, 6, 64
    tab, rope = make((16, 0, 0), offset=32, half=half)
    big = draw((heads, tokens, dim + lead + tail), dtype, 3)
    x = big.transpose(0, 1)[:, :, lead:lead + dim]
    pos = torch.arange(tokens, dtype=torch.int32)[:, None]
    out = torch.full((tokens, heads + 1, dim + lead + tail), 7.0, dtype=dtype, device="cuda")
    y = out[:, :heads, lead:lead + dim]
    bigd = big.cuda()
    V.mla_rope_apply(rope, bigd.transpose(0, 1)[:, :, lead:lead + dim], pos.cuda(), y)
    check(x, y, tab, rope, pos, half, 32)
    assert (out[:, heads] == 7).all() and (out[:, :, :lead] == 7).all()
    assert (out[:, :, lead + dim:] == 7).all()


def test_gradient_is_the_inverse():
    """The inverse is the transposed map: <R x, g> = <x, R' g>, and the slope
    of <R x, g> along a direction, taken by differences, is <R' g, d>. The map
    is linear, so differences carry only fp32 rounding: sums of 8 x 4 x 64
    products of size about 1 with relative error 2^-22 each."""
    tab, rope = make((32, 0, 0), half=True, scaling=3, factor=4.0)
    x, g, d = (draw((8, 4, 64), torch.float32, s).cuda() for s in (1, 2, 3))
    pos = torch.arange(8, dtype=torch.int32, device="cuda")[:, None] * 31

    def fwd(v):
        y = torch.empty_like(v)
        V.mla_rope_apply(rope, v, pos, y)
        return (y.double() * g.double()).sum().item()

    dx = torch.empty_like(g)
    V.mla_rope_apply(rope, g, pos, dx, inverse=True)
    tol = 2048 * 2.0 ** -22 * 4
    assert abs(fwd(x) - (x.double() * dx.double()).sum().item()) <= tol
    slope = (fwd(x + 0.5 * d) - fwd(x - 0.5 * d))
    assert abs(slope - (dx.double() * d.double()).sum().item()) <= 2 * tol


def test_positions_are_checked_and_bytes_past_4_gib():
    tab, rope = make((16, 0, 0), length=8)
    x = draw((3, 1, 32), torch.float32, 1)
    pos = torch.tensor([[0], [8], [-1]], dtype=torch.int32)
    y = torch.empty_like(x, device="cuda")
    V.mla_rope_apply(rope, x.cuda(), pos.cuda(), y)
    assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE
    assert torch.equal(y.cpu(), x)                    # position 0 turns nothing
    big = torch.zeros(2, (1 << 31) + 64, dtype=torch.bfloat16, device="cuda")  # 8 GiB
    v = big[:, -32:].unsqueeze(1)
    v.copy_(draw((2, 1, 32), torch.bfloat16, 2))
    src = v.cpu()
    V.mla_rope_apply(rope, v, torch.tensor([[3], [5]], dtype=torch.int32, device="cuda"), v)
    check(src, v, tab, rope, torch.tensor([[3], [5]]), False, 0)


def test_side_stream_and_empty():
    tab, rope = make((6, 5, 5))
    x = draw((50, 12, 32), torch.bfloat16, 4)
    pos = torch.randint(0, 300, (50, 3), dtype=torch.int32)
    xd, pd = x.cuda(), pos.cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = torch.empty_like(xd)
    V.mla_rope_apply(rope, xd, pd, y, stream=s)
    s.synchronize()
    check(x, y, tab, rope, pos, False, 0)
    V.mla_rope_apply(rope, xd[:0], pd[:0], y[:0])


def test_refusals():
    tab, rope = make((6, 5, 5))
    x = torch.zeros(4, 2, 32, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        V.mla_rope_apply(rope, x.cpu(), pos, x)
    with pytest.raises(TypeError):
        V.mla_rope_apply(rope, x, pos, x.float())
    with pytest.raises(ValueError):
        V.mla_rope_apply(rope, x, pos[:, :1], x)
    with pytest.raises(ValueError):
        V.mla_rope_apply(rope, x.transpose(1, 2), pos, x.transpose(1, 2))
    with pytest.raises(V.MlaError) as e:              # 32 rotated channels in a head of 16
        V.mla_rope_apply(rope, x[:, :, :16], pos, x[:, :, :16])
    assert e.value.code == V.MLA_ERR_ARG
