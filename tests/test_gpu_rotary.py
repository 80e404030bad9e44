"""Rotary positions and their gradient against pairs of channels as complex numbers in 64 bits."""
import pytest
import torch

import paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    import paper_2509_24663_amd as m
    m.lib()
    return m


def _tol(dtype, want):
    # bf16: the result's own rounding; fp32: cos and sin to 2e-7 of their magnitude (angle 7e-10, series, rounding), two products and a sum of values
    # of at most 6 in 32 bits: below 6 * (2e-7 + 3 * 2^-24) * 2
    return (2.0 ** -8 * want.abs() + 6e-6) if dtype == "bf16" else torch.full_like(want, 6e-6)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype,d,rot_dim,heads,tokens", [
    ("bf16", 128, 128, 32, 1), ("bf16", 128, 104, 3, 77), ("bf16", 64, 32, 4, 130), ("bf16", 64, 2, 1, 5), ("bf16", 128, 50, 2, 33),
    ("fp32", 64, 64, 8, 19), ("fp32", 128, 40, 5, 64), ("fp32", 64, 8, 6, 1), ("bf16", 128, 128, 32, 9000)])
def test_rotary_and_gradient(m, layout, dtype, d, rot_dim, heads, tokens):
    p = m.Params.make(dtype, heads, heads, d)
    freq = paged.frequencies(rot_dim)
    rot = m.Rotary(m.rotary_turns(rot_dim), rot_dim, layout, 1.25)
    gen = torch.Generator(device="cuda").manual_seed(7)
    # heads of packed projections: a view with other strides
    wide = torch.randn((tokens, heads + 2, d), generator=gen, device="cuda").clamp(-4, 4).to(p.torch_dtype)
    x = wide[:, 1:heads + 1]
    pos = torch.randint(-3, 1 << 20, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    want = paged.turned(x, pos, freq, layout, 1.25)
    got = m.rotary_fwd(p, rot, x, pos)
    assert bool(((got.double() - want).abs() <= _tol(dtype, want)).all())
    back = paged.turned(x, pos, freq, layout, 1.25, back=True)
    grad = m.rotary_bwd(p, rot, x, pos)
    assert bool(((grad.double() - back).abs() <= _tol(dtype, back)).all())
    # in place, and into a strided output: the same bits, the heads beside it untouched
    there = wide.clone()
    m.rotary_fwd(p, rot, there[:, 1:heads + 1], pos, out=there[:, 1:heads + 1])
    assert torch.equal(there[:, 1:heads + 1], got)
    assert torch.equal(there[:, 0], wide[:, 0]) and torch.equal(there[:, -1], wide[:, -1])
    # head-major rows
    turned = m.rotary_fwd(p, rot, x.transpose(0, 1).contiguous().transpose(0, 1), pos)
    assert torch.equal(turned, got)


def test_gradient_against_differences(m):
    """y is linear in x: <dy, y(x + e) - y(x)> = <bwd(dy), e> for steps of any size."""
    p = m.Params.make("fp32", 2, 2, 64)
    rot = m.Rotary(m.rotary_turns(24), 24, "half", 0.5)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, e, dy = (torch.randn((41, 2, 64), generator=gen, device="cuda") for _ in range(3))
    pos = torch.arange(41, device="cuda", dtype=torch.int32) * 1000
    diff = m.rotary_fwd(p, rot, x + e, pos).double() - m.rotary_fwd(p, rot, x, pos).double()
    left, right = (dy.double() * diff).sum(), (m.rotary_bwd(p, rot, dy, pos).double() * e.double()).sum()
    # 5248 products of values of about 1, each off by at most 1e-6
    assert abs(float(left - right)) <= 5248 * 1e-6


def test_far_positions_are_exact(m):
    """At position 2^31 - 1 an angle in 32 bits would be off by hundreds of radians."""
    p = m.Params.make("fp32", 1, 1, 128)
    turns = m.rotary_turns(128)
    rot = m.Rotary(turns, 128)
    pos = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345], dtype=torch.int32, device="cuda")
    x = torch.zeros((3, 1, 128), device="cuda")
    x[..., :64] = 1
    got = m.rotary_fwd(p, rot, x, pos)[:, 0]
    for i, t in enumerate(pos.tolist()):
        for j, f in enumerate(turns.tolist()):
            frac = ((t * (f % 2 ** 64)) % 2 ** 64) / 2 ** 64           # exact integers, rounded once
            a = torch.tensor(2 * torch.pi * frac, dtype=torch.float64)
            assert abs(float(got[i, j]) - float(a.cos())) <= 3e-7 and abs(float(got[i, 64 + j]) - float(a.sin())) <= 3e-7


def test_nothing_to_turn(m):
    p = m.Params.make("bf16", 2, 2, 64)
    rot = m.Rotary(m.rotary_turns(64), 64)
    x = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert m.rotary_fwd(p, rot, x, torch.empty(0, dtype=torch.int32, device="cuda")).shape == (0, 2, 64)
