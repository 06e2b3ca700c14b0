"""The plain forms that the tests of the operators around the attention compare
with, on the CPU: gradients against differences, codes against torch's own
conversion, the cache's offsets against each other."""
import torch

import around_reference as ref


def test_gradients_against_differences():
    g = torch.Generator().manual_seed(0)
    x = torch.randn(1, 2, 5, 64, generator=g, dtype=torch.float64)
    gain = 1 + 0.3 * torch.randn(64, generator=g, dtype=torch.float64)
    angle = torch.randn(1, 5, 24, generator=g, dtype=torch.float64)
    cs = (angle.cos(), angle.sin())
    dy = torch.randn(x.shape, generator=g, dtype=torch.float64)
    for halves in (False, True):
        for eps in (0.0, 1e-6):
            w = gain if eps else None
            dx, dgain, _, _ = ref.rope_backward(x, w, eps, cs, halves, dy)
            value = lambda a, b: (ref.rope_forward(None, a, b, eps, cs, halves)[0] * dy).sum()
            way = torch.randn(x.shape, generator=g, dtype=torch.float64)
            step = 1e-5
            slope = (value(x + step * way, w) - value(x - step * way, w)) / (2 * step)
            assert abs(slope - (dx * way).sum()) <= 1e-7 * (dx.abs() * way.abs()).sum()
            if eps:
                to = torch.randn(64, generator=g, dtype=torch.float64)
                slope = (value(x, w + step * to) - value(x, w - step * to)) / (2 * step)
                assert abs(slope - (dgain * to).sum()) <= 1e-7 * (dgain.abs() * to.abs()).sum()


def test_codes_against_torch():
    x = torch.randn(4000, generator=torch.Generator().manual_seed(1)) * torch.logspace(-4, 2, 4000)
    x = torch.cat([x.clamp(-448, 448), ref.VALUES[:127].float(), -ref.VALUES[:127].float(),
                   ((ref.VALUES[1:127] + ref.VALUES[:126]) / 2).float()])
    assert torch.equal(ref.e4m3_codes(x.double()).to(torch.uint8), x.to(torch.float8_e4m3fn).view(torch.uint8))
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double()
    assert torch.equal(torch.nan_to_num(ref.VALUES, nan=-1.0), torch.nan_to_num(want, nan=-1.0))


def test_the_power_is_the_smallest():
    x = torch.tensor([[1.75], [1.7500001], [1.0], [448.0], [0.0], [2.0 ** -90], [3.0e38]], dtype=torch.float32)
    assert ref.quantised(x)[1].tolist() == [-8, -7, -8, 0, -100, -98, 120]


def test_every_byte_of_a_page_has_one_place():
    for D in (64, 128):
        seen = torch.zeros(128 * D + 128, dtype=torch.int64)
        for j in range(64):
            k, v, ke, ve = ref.offsets(j, D)
            for at in (k, v, torch.tensor([ke]), torch.tensor([ve])):
                seen[at] += 1
        assert (seen == 1).all()


def test_places_are_the_cube_major_order():
    import numpy as np

    from workload import Problem, raster_to_cube_major
    p = Problem(1, 1, 1, 8, 5, 6, 7)
    x = torch.arange(1, 5 * 6 * 7 + 1).float()[:, None].expand(-1, 8)
    places, _, L = ref.place_of(p)
    want = torch.from_numpy(raster_to_cube_major(np.ascontiguousarray(x.numpy()), p))
    assert L == p.L and torch.equal(ref.to_places(x[None, None], places, L)[0, 0], want)
