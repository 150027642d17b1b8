"""States of gas_adamw_steps bit for bit against their definition in float32, where every product and sum is rounded by itself: what a compiler
fuses moves a value past the line between two codes now and then, a whole code."""
import numpy as np
import pytest
import torch

import paper_2106_05609_amd as gas

pytestmark = pytest.mark.gpu
F = np.float32
HYPER = dict(beta1=0.9, beta2=0.999, eps=1e-8)


def dice(total, step):
    """Two numbers of 16 bits of every element, by its place and the step (places below 2^32)."""
    x = np.arange(total, dtype=np.uint64).astype(np.uint32) ^ np.uint32(step * 0x9E3779B9 & 0xFFFFFFFF)
    with np.errstate(over="ignore"):
        x = (x ^ (x >> np.uint32(16))) * np.uint32(0x7FEB352D)
        x = (x ^ (x >> np.uint32(15))) * np.uint32(0x846CA68B)
    x = x ^ (x >> np.uint32(16))
    return x & np.uint32(0xFFFF), x >> np.uint32(16)


def moments(m, v, g):
    return m * F(0.9) + g * F(1.0 - 0.9), v * F(0.999) + g * g * F(1.0 - 0.999)


def coded(a, power, top, die):
    """(scales, codes) of non-negative values in blocks of 256."""
    a = a.reshape(-1, 256)
    scale = a.max(1, keepdims=True)
    scale = np.where(scale < np.finfo(F).tiny, F(0), scale)
    with np.errstate(divide="ignore"):
        x = a * np.where(scale > 0, F(1) / scale, F(0)) * F(top ** power)
    r = np.sqrt(x) if power == 2 else np.sqrt(np.sqrt(x))
    k = np.minimum(np.floor(r), F(top - 1))
    low, up = k * k, (k + F(1)) * (k + F(1))
    if power == 4:
        low, up = low * low, up * up
    more = (die.reshape(-1, 256).astype(F) + F(0.5)) * F(1 / 65536) * (up - low) < x - low
    return scale[:, 0], (k + more).astype(np.int32)


def decoded(k, v, scales):
    k, v = k.astype(F).reshape(-1, 256), v.astype(F).reshape(-1, 256)
    t = v * v * F(1 / 65025)
    return (scales[:, :1] * (k * np.abs(k) * F(1 / 16129))).reshape(-1), (scales[:, 1:] * t * t).reshape(-1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("spread", [0.0, 1.0, 3.0])
def test_states_by_the_definition_in_32_bits(bits, spread):
    n = 256 * 8192
    gen = torch.Generator().manual_seed(11)
    total = gas.gas_adamw_elements([n])
    new = lambda dt: torch.zeros(total, dtype=dt, device="cuda")
    w = torch.zeros(n, device="cuda")
    m, v = (new(torch.float32), new(torch.float32)) if bits == 32 else (new(torch.int8), new(torch.uint8))
    scales = None if bits == 32 else torch.zeros(total // 256, 2, device="cuda")
    want_m, want_v = np.zeros(n, F), np.zeros(n, F)
    for t in (1, 2, 3):
        g = (torch.randn(n, generator=gen) * torch.exp(spread * torch.randn(n, generator=gen)) * 1e-4)
        gas.gas_adamw_steps([w], [g.cuda()], m, v, 1e-3, t, scales=scales, **HYPER)
        want_m, want_v = moments(want_m, want_v, g.numpy())
        if bits == 32:
            assert np.array_equal(m.cpu().numpy(), want_m) and np.array_equal(v.cpu().numpy(), want_v), t
            continue
        dm, dv = dice(n, t)
        sm, km = coded(np.abs(want_m), 2, 127, dm)
        sv, kv = coded(want_v, 4, 255, dv)
        kv = np.where((kv == 0) & (want_v.reshape(-1, 256) > 0) & (sv[:, None] > 0), 1, kv)
        km = np.where(want_m.reshape(-1, 256) < 0, -km, km)
        got = scales.cpu().numpy()
        assert np.array_equal(got, np.stack([sm, sv], 1)), t
        assert np.array_equal(m.cpu().numpy().reshape(-1, 256), km), t
        assert np.array_equal(v.cpu().numpy().reshape(-1, 256), kv), t
        want_m, want_v = decoded(m.cpu().numpy(), v.cpu().numpy(), got)
