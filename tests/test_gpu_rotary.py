"""Rotary positions against the rotation of complex numbers in 64 bits.

Cosine and sine are off by at most 2^-21 (up to position 2^24: the angle's 64-bit product is off by 2^-52 of up to 2^22 turns, 2^-30 turns; the
reduced angle is narrowed to 24 bits of up to pi, and CUDA's sincospif is off by at most a step, together below 2^-22); a result is two products and
a sum in fp32, 3 * 2^-24 of |a| + |b|, and one rounding to the type."""
import numpy as np
import pytest

from oracle import prompt_oracle as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device; the library has no CPU path")
    from paper_2510_01565_b200 import binding, build
    build.build_library()
    binding.load_library()
    return binding


def check(got, x, positions, heads, rotary, interleaved, base=10000.0, factor=1.0, ramp=None, magnitude=1.0, inverse=False):
    import torch
    xd = x.double().cpu().numpy()
    freq = P.frequencies(rotary, base, factor, ramp)
    want = P.rotary(xd, positions, heads, freq, interleaved, magnitude, inverse)
    size = np.abs(xd).reshape(xd.shape[0], heads, -1)
    both = size.copy()                            # |a| + |b| of a channel's pair
    n = rotary // 2
    ia, ib = (np.arange(0, rotary, 2), np.arange(1, rotary, 2)) if interleaved else (np.arange(n), np.arange(n, rotary))
    both[:, :, ia] = both[:, :, ib] = size[:, :, ia] + size[:, :, ib]
    info = torch.finfo(x.dtype)
    tol = magnitude * both.reshape(xd.shape) * (2.0 ** -21 + 4 * 2.0 ** -24)
    tol = tol + (np.abs(want) + tol) * info.eps / 2 + info.smallest_normal * info.eps / 2
    assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()
    kept = x.reshape(x.shape[0], heads, -1)[:, :, rotary:]
    assert torch.equal(got.reshape(x.shape[0], heads, -1)[:, :, rotary:], kept)


def spread(lens, first):
    return np.concatenate([np.arange(f, f + l) for l, f in zip(lens, first)] or [np.empty(0)])


CASES = [([1], [0], 1, 64, 64), ([1, 1, 1], [7, 131071, 16777215], 40, 128, 128), ([5, 0, 130], [0, 9, 1000], 3, 80, 80), ([77], [3], 12, 64, 32),
         ([300, 41], [0, 0], 5, 96, 48), ([2, 3], [10, 20], 2, 6, 4), ([6000], [0], 2, 128, 128), ([33], [5], 7, 256, 256), ([9], [1], 3, 40, 20),
         ([5], [0], 2, 300, 254), ([4], [2], 1, 2, 2)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("lens,first,heads,dim,rotary", CASES)
def test_rotation(B, lens, first, heads, dim, rotary, kind, interleaved):
    import torch
    x = torch.randn(sum(lens), heads * dim, generator=torch.Generator().manual_seed(dim)).to(getattr(torch, kind)).cuda()
    got = B.dit_rotary(x, heads, lens, first=first, rotary_dim=rotary, interleaved=interleaved)
    check(got, x, spread(lens, first), heads, rotary, interleaved)
    places = torch.from_numpy(spread(lens, first).astype(np.int32)).cuda()
    assert torch.equal(got, B.dit_rotary(x, heads, positions=places, rotary_dim=rotary, interleaved=interleaved))


@pytest.mark.parametrize("factor,ramp,base,magnitude", [(8.0, None, 10000.0, 1.0), (8.0, (1, 4, 8192), 500000.0, 1.0), (40.0, (1.0, 32.0, 4096), 10000.0, 1.37)])
def test_scaled_for_longer_contexts(B, factor, ramp, base, magnitude):
    import torch
    x = torch.randn(600, 4 * 128, generator=torch.Generator().manual_seed(1)).cuda()
    got = B.dit_rotary(x, 4, [600], first=[120000], base=base, factor=factor, ramp=ramp, magnitude=magnitude)
    check(got, x, spread([600], [120000]), 4, 128, False, base, factor, ramp, magnitude)


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_inverse_is_the_transposed_map(B, interleaved):
    """<rotary(x), g> = <x, inverse(g)>: the gradient of a rotation, and a difference quotient of it."""
    import torch
    g = torch.Generator().manual_seed(4)
    x, grad, step = (torch.randn(50, 3 * 64, generator=g).cuda() for _ in range(3))
    kw = dict(first=[1000], rotary_dim=32, interleaved=interleaved, magnitude=1.5, factor=2.0)
    back = B.dit_rotary(grad, 3, [50], inverse=True, **kw)
    left = (B.dit_rotary(x, 3, [50], **kw).double() * grad.double()).sum()
    right = (x.double() * back.double()).sum()
    scale = (x.double().abs() * grad.double().abs()).sum()
    assert abs(left - right) <= 4 * 2.0 ** -20 * 1.5 * scale
    moved = (B.dit_rotary(x + step, 3, [50], **kw).double() - B.dit_rotary(x, 3, [50], **kw).double()) * grad.double()
    size = ((x.abs() + step.abs()).double() * grad.double().abs()).sum()
    assert abs(moved.sum() - (step.double() * back.double()).sum()) <= 8 * 2.0 ** -20 * 1.5 * size
    again = B.dit_rotary(B.dit_rotary(x, 3, [50], interleaved=interleaved), 3, [50], inverse=True, interleaved=interleaved)
    assert (again - x).abs().max() <= 8 * 2.0 ** -21 * x.abs().max()


@pytest.mark.parametrize("kind", ["float16", "float32"])
def test_strides_in_place_and_surroundings(B, kind):
    import torch
    kind = getattr(torch, kind)
    for left, heads, dim, interleaved in ((0, 6, 64, False), (8, 4, 64, True), (3, 4, 64, False), (1, 3, 10, True)):
        big = torch.randn(90, heads * dim + left + 5, generator=torch.Generator().manual_seed(left)).to(kind).cuda()
        before = big.clone()
        x = big[2:-3, left:left + heads * dim]
        rotary = dim // 2 // 2 * 2
        apart = B.dit_rotary(x, heads, [85], first=[11], rotary_dim=rotary, interleaved=interleaved)
        check(apart, x, spread([85], [11]), heads, rotary, interleaved)
        same = B.dit_rotary(x, heads, [85], first=[11], rotary_dim=rotary, interleaved=interleaved, out=x)
        assert same.data_ptr() == x.data_ptr() and torch.equal(x, apart)
        big[2:-3, left:left + heads * dim] = before[2:-3, left:left + heads * dim]
        assert torch.equal(big, before)


def test_positions_of_any_sign_and_values_that_are_no_numbers(B):
    import torch
    places = torch.tensor([-5, 2 ** 31 - 1, -2 ** 31, 0], dtype=torch.int32, device="cuda")
    x = torch.randn(4, 64, generator=torch.Generator().manual_seed(2)).cuda()
    got = B.dit_rotary(x, 1, positions=places)
    check(got[[0, 3]], x[[0, 3]], [-5, 0], 1, 64, False)
    want = P.rotary(x.double().cpu().numpy(), places.cpu().numpy(), 1, P.frequencies(64))
    assert np.abs(got.double().cpu().numpy() - want).max() < 1e-5      # 2^31 * 2^-53 turns: 2^-22, beside the bound above
    x[1, 3], x[2, 40] = float("inf"), float("nan")
    got = B.dit_rotary(x, 1, positions=torch.ones(4, dtype=torch.int32, device="cuda"))
    odd = ~torch.isfinite(got)
    assert odd.nonzero().tolist() == [[1, 3], [1, 35], [2, 8], [2, 40]]


def test_empty(B):
    import torch
    assert B.dit_rotary(torch.empty(0, 128, device="cuda"), 2, []).shape == (0, 128)
    assert B.dit_rotary(torch.empty(0, 128, device="cuda"), 2, [0, 0], first=[3, 4]).shape == (0, 128)
    assert B.dit_rotary(torch.empty(0, 128, device="cuda"), 2, positions=torch.empty(0, dtype=torch.int32, device="cuda")).shape == (0, 128)
