"""Rotary positions at their limits: the phase of far positions, where a column shows it to its last bits, and the differentiable calls without keys."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from tests import rotary_reference as R

pytestmark = pytest.mark.gpu

PI = Fraction(314159265358979323846264338327950288419716939937510582097494459230781640628620899, 10 ** 80)


@pytest.fixture(scope="module")
def mala():
    from paper_2609_32712_b200 import mala as m
    m.lib()
    return m


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _near_whole_turns(f, end, step):
    """Positions from `end` on, `step` by `step`, at which f radians per position come within 2^-20 of a whole turn: (position, phase in turns, exact)."""
    turns = Fraction(f) / (2 * PI)
    unit = round((turns - round(turns)) * 2 ** 64) % 2 ** 64
    found = []
    for x0 in range(0, 1 << 24, 1 << 20):
        pos = end + step * np.arange(x0, x0 + (1 << 20), dtype=np.int64)
        phase = (pos.astype(np.uint64) * np.uint64(unit)).view(np.int64)
        for p in pos[np.abs(phase) < 2 ** 44].tolist():
            exact = turns * p
            exact = float(exact - round(exact))
            if 2.0 ** -24 < abs(exact) < 2.0 ** -20:
                found.append((p, exact))
        if len(found) >= 4:
            return found[:4]
    raise AssertionError("no such positions")


@pytest.mark.parametrize("end,step", [(2 ** 31 - 1, -1), (-2 ** 31, 1), (2 ** 30, 1)])
@pytest.mark.parametrize("pair", [1, 3])
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_phases(mala, end, step, pair, interleaved):
    """Angles are exact to 2^-31 turns at any position: near whole turns the sine is the phase itself, and bf16 shows it to 2^-8 of its value."""
    d = 128
    f, _ = mala.rotary_frequencies(d, 500000.0)
    rot = mala.Rotary(f, interleaved=interleaved)
    at = _near_whole_turns(f[pair].item(), end, step)
    pos = _i32([p for p, _ in at])
    first, second = (2 * pair, 2 * pair + 1) if interleaved else (pair, pair + d // 2)
    q = torch.zeros((1, len(at), 1, d), dtype=torch.bfloat16, device="cuda")
    q[..., first] = 1
    k = torch.zeros_like(q)
    pages = torch.zeros((1, 16, 1, d), dtype=torch.bfloat16, device="cuda")
    outs = [mala.rotary(q, None, rot, positions=pos[None])[0][0, :, 0]]
    slots = torch.arange(len(at), device="cuda")
    outs.append(mala.rotary_write(k[0], q[0], k[0], pos, slots, pages, torch.zeros_like(pages), rot)[:, 0] + pages[0, :len(at), 0])
    for out in outs:
        for (_, phase), y in zip(at, out.double()):
            want = math.sin(2 * math.pi * phase)
            # 2^-31 turns; fp32's roundings of phase and series (2^-21 of a sine this small); half a step of bf16
            assert abs(y[second].item() - want) <= 2 * math.pi * 2.0 ** -31 + abs(want) * (2.0 ** -8 + 2.0 ** -21), (phase, y[second].item() / want)
            assert y[first].item() == 1.0


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("normed", [False, True])
def test_gradients_without_keys(mala, packed, normed):
    from paper_2609_32712_b200 import autograd as A
    d, total = 64, 9
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn((1, total, 3, d), generator=g, device="cuda").to(torch.bfloat16).requires_grad_()
    w = (torch.randn(d, generator=g, device="cuda") * 0.3 + 1).requires_grad_() if normed else None
    rot, eps = mala.Rotary(mala.rotary_frequencies(48)[0]), 1e-5 if normed else None
    cu = _i32([0, 4, 9])
    if packed:
        out, keys = A.rotary_packed(q, None, cu, cu, rot, q_weight=w, eps=eps)
        pos = torch.tensor([0, 1, 2, 3, 0, 1, 2, 3, 4], device="cuda")[None]
    else:
        out, keys = A.rotary(q, None, rot, q_weight=w, eps=eps)
        pos = torch.arange(total, device="cuda")[None]
    assert keys is None
    dy = torch.randn(q.shape, generator=g, device="cuda").to(torch.bfloat16)
    out.backward(dy)
    a = (pos, rot.inv_freq, False, 1.0, eps, w.detach() if normed else None)
    dx, dw, total_w = R.backward(dy, q.detach(), *a)
    size = R.backward_size(dy, q.detach(), *a)
    # (tolerances of the calls with keys: half a step of bf16, 2^-19 of the terms before it; fp32 sums of 27 terms)
    assert ((q.grad.double() - dx).abs() <= 2.0 ** -8 * dx.abs() + 2.0 ** -19 * size).all()
    if normed:
        assert ((w.grad.double() - dw).abs() <= total_w * (2.0 ** -19 + 40 * 2.0 ** -24)).all()
