"""gas_sq_norms, gas_adamw_steps and gas_adamw_unpack against their definitions in 64 bits (tests/residual_reference.py)."""
import numpy as np
import pytest
import torch

import paper_2106_05609_amd as gas
from tests import residual_reference as R

pytestmark = pytest.mark.gpu
SIZES = [1, 2, 255, 256, 257, 0, 1000, 4096, 64, 47 * 33, 65_537, 3]
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8)


def model(sizes, dtypes, bits, master, seed=0, offset=0, scale=1e-2):
    """Tensors (each `offset` elements into memory of its own), gradients and the state on the GPU."""
    gen = torch.Generator().manual_seed(seed)
    r = lambda n: torch.randn(n, generator=gen)
    put = lambda v, dt: torch.cat([torch.zeros(offset), v]).to(dt).cuda()[offset:]
    dtypes = [dtypes[i % len(dtypes)] for i in range(len(sizes))]
    s = dict(ws=[put(r(n) * 0.1, dt) for n, dt in zip(sizes, dtypes)], gs=[put(r(n) * scale * torch.exp(r(n)), torch.float32) for n in sizes])
    total = gas.gas_adamw_elements(sizes)
    assert total == R.layout(sizes)[1]
    new = lambda dt: torch.zeros(total, dtype=dt, device="cuda")
    s.update(m=new(torch.float32 if bits == 32 else torch.int8), v=new(torch.float32 if bits == 32 else torch.uint8),
             scales=None if bits == 32 else torch.zeros(total // 256, 2, device="cuda"), master=new(torch.float32) if master else None)
    if master:
        for w, at in zip(s["ws"], R.layout(sizes)[0]):
            s["master"][at:at + w.numel()] = w.float() + 1e-4 * r(w.numel()).cuda()
    return s


def step(s, **kw):
    gas.gas_adamw_steps(s["ws"], s["gs"], s["m"], s["v"], scales=s["scales"], master=s["master"], **{**HYPER, **kw})


def values(s):
    """What the state stands for, float64."""
    if s["scales"] is None:
        return s["m"].double().cpu().numpy(), s["v"].double().cpu().numpy()
    return R.decode(s["m"].cpu().numpy(), s["v"].cpu().numpy(), s["scales"].cpu().numpy())


def check_step(s, t, c=1.0, wd=None, **kw):
    """One step, checked: weights and 32-bit states to a few last places of what they are summed from, codes to their neighbours."""
    sizes = [w.numel() for w in s["ws"]]
    starts = R.layout(sizes)[0]
    m0, v0 = values(s)
    w0 = [w.double().cpu().numpy() for w in s["ws"]]
    if s["master"] is not None:
        master = s["master"].double().cpu().numpy()
        w0 = [master[at:at + len(w)] if x.dtype == torch.bfloat16 else w for w, x, at in zip(w0, s["ws"], starts)]
    step(s, **{**dict(step=t, weight_decay=0.0 if wd is None else wd), **kw})
    m1, v1 = values(s)
    wd = [wd or 0.0] * len(sizes) if not isinstance(wd, list) else wd
    h = HYPER
    for i, (at, n) in enumerate(zip(starts, sizes)):
        g, part = s["gs"][i].double().cpu().numpy(), slice(at, at + n)
        w, m, v = R.adamw(w0[i], g, m0[part], v0[part], h["lr"], t, h["beta1"], h["beta2"], h["eps"], wd[i], c)
        change = np.abs(w - w0[i]) + np.abs(w0[i]) * h["lr"] * wd[i]
        got = s["ws"][i].double().cpu().numpy()
        half = s["ws"][i].dtype == torch.bfloat16
        # |w| rounds once or twice, the change is a chain of some ten operations
        allowed = 3 * R.EPS32 * np.abs(w) + 32 * R.EPS32 * change
        if half and s["master"] is not None:
            kept = s["master"][part].double().cpu().numpy()
            assert (np.abs(kept - w) <= allowed).all()
            assert torch.equal(s["master"][part].bfloat16(), s["ws"][i])
        else:
            assert (np.abs(got - w) <= allowed + (R.EPS16 * np.abs(w) * 1.001 if half else 0)).all(), i
        gc = np.abs(g) * c
        if s["scales"] is None:
            assert (np.abs(m1[part] - m) <= 4 * R.EPS32 * (np.abs(m0[part]) + gc)).all()
            assert (np.abs(v1[part] - v) <= 6 * R.EPS32 * v + 1e-45).all()
            continue
        pad = lambda z: np.concatenate([z, np.zeros(-len(z) % 256)]).reshape(-1, 256)
        for got_, want, top, power in ((m1, np.abs(m), 127, 2), (v1, v, 255, 4)):
            largest = pad(want).max(1, keepdims=True)
            near = pad(np.abs(got_[part]))
            rel = np.divide(pad(want), largest, out=np.zeros_like(near), where=largest > 0)
            k = np.floor(rel ** (1 / power) * top * (1 - 1e-6))
            low, up = largest * (k / top) ** power, largest * (np.minimum(k + 2, top) / top) ** power
            assert (near >= low * (1 - 1e-5)).all() and (near <= up * (1 + 1e-5)).all()
        big = np.abs(m) > np.repeat(pad(np.abs(m)).max(1), 256)[:n] * 1e-3
        assert (np.sign(m1[part][big]) == np.sign(m[big])).all()
        assert (v1[part][v > 1e-37] > 0).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtypes,master", [(["f32"], False), (["bf16"], False), (["bf16"], True), (["bf16", "f32"], True), (["f32", "bf16"], False)])
@pytest.mark.parametrize("offset", [0, 1])
def test_steps(bits, dtypes, master, offset):
    dts = [dict(f32=torch.float32, bf16=torch.bfloat16)[d] for d in dtypes]
    s = model(SIZES, dts, bits, master, offset=offset)
    wd = [0.0 if i % 3 else 0.1 for i in range(len(SIZES))]
    for t in (1, 2, 3):
        check_step(s, t, wd=wd)
    check_step(s, 1000, wd=0.05)
    # what pads the tensors to 256 stays zero
    starts, total = R.layout(SIZES)
    held = np.zeros(total, bool)
    for at, n in zip(starts, SIZES):
        held[at:at + n] = True
    for x in (s["m"], s["v"]) + ((s["master"],) if master else ()):
        assert (x.cpu().numpy()[~held] == 0).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_a_launch_takes(bits):
    check_step(model([(37 * i) % 700 for i in range(300)], [torch.float32, torch.bfloat16], bits, True), 5, wd=0.01)


def test_a_tensor_given_twice_is_updated_twice():
    s = model([300, 300], [torch.float32], 32, False)
    s["ws"][1] = s["ws"][0]
    one = [s["ws"][0].clone()]
    a, b = model([300], [torch.float32], 32, False), model([300], [torch.float32], 32, False)
    for other, g in ((a, s["gs"][0]), (b, s["gs"][1])):
        other["ws"], other["gs"] = one, [g]
        step(other, step=1)
    step(s, step=1)
    assert torch.equal(s["ws"][0], one[0])


@pytest.mark.parametrize("bits", [32, 8])
def test_clipping_and_steps_on_the_device(bits):
    s = model([1000, 64 * 64], [torch.float32], bits, False)
    sq, steps = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for t in (1, 2, 3):
        gas.gas_sq_norms(s["gs"], sq, steps=steps)
        assert steps.item() == t
        norm = np.sqrt(sum(g.double().square().sum().item() for g in s["gs"]))
        check_step(s, t, c=min(1.0, 0.3 / (norm + 1e-6)), step=0, steps=steps, sq_norm=sq, max_norm=0.3)
    check_step(s, 4, step=4, sq_norm=sq)                              # no bound: not clipped
    check_step(s, 5, step=5, sq_norm=sq, max_norm=norm * 2)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), -float("inf"), 3e38])
def test_a_step_with_an_infinity_changes_nothing(bits, bad):
    s = model([1000, 300], [torch.float32, torch.bfloat16], bits, True)
    step(s, step=1)
    keep = [x.clone() for x in s["ws"] + [y for y in (s["m"], s["v"], s["scales"], s["master"]) if y is not None]]
    s["gs"][1][17] = bad                                             # 3e38 squared is past float32 too
    sq, steps = torch.zeros(1, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    gas.gas_sq_norms(s["gs"], sq, steps=steps)
    step(s, steps=steps, sq_norm=sq, max_norm=1.0)
    assert steps.item() == 1 and not torch.isfinite(sq).item()
    for x, y in zip(keep, s["ws"] + [y for y in (s["m"], s["v"], s["scales"], s["master"]) if y is not None]):
        assert torch.equal(x, y)


def test_eight_bits_without_a_norm_keep_an_infinity_in_its_block():
    s = model([1024], [torch.float32], 8, False)
    s["gs"][0][300] = float("nan")
    step(s, step=1)
    m, v = values(s)
    assert np.isnan(m[256:512]).all() and np.isnan(v[256:512]).all()
    assert np.isfinite(np.delete(m, np.arange(256, 512))).all() and np.isfinite(np.delete(v, np.arange(256, 512))).all()


@pytest.mark.parametrize("scale", [1e-18, 1e-21, 1e-30, 1e15])
def test_eight_bits_of_very_small_and_very_large_gradients(scale):
    """v's largest near, below and far below the smallest normal number, and near the largest."""
    s = model([512], [torch.float32], 8, False, scale=scale)
    for t in (1, 2):
        step(s, step=t)
        m, v = values(s)
        assert np.isfinite(m).all() and np.isfinite(v).all() and torch.isfinite(s["ws"][0]).all()
    if scale == 1e-18:
        check_step(s, 3)


def test_eight_bits_round_to_the_expectation():
    """The mean of what a value becomes, over many places, is the value: a code is at most q wide there, so the mean of n is off by less
    than 5 q / (2 sqrt(n)) but once in a million."""
    n = 256 * 4096
    m_in = 0.013                                                     # beside a largest of 1
    s = model([n], [torch.float32], 8, False)
    g = torch.full((n // 256, 256), m_in, device="cuda")
    g[:, 0] = 1.0
    s["gs"] = [g.view(-1)]
    step(s, step=1, beta1=0.0, beta2=0.0)
    m, v = (z.reshape(-1, 256)[:, 1:] for z in values(s))
    k = np.floor(np.sqrt(m_in) * 127)
    width = ((k + 1) ** 2 - k ** 2) / 127 ** 2
    assert abs(m.mean() - m_in) <= 5 * width / (2 * np.sqrt(m.size)) + 1e-6 * m_in
    k = np.floor(np.sqrt(m_in) * 255)                                # v = g^2
    width = ((k + 1) ** 4 - k ** 4) / 255 ** 4
    assert abs(v.mean() - m_in ** 2) <= 5 * width / (2 * np.sqrt(v.size)) + 1e-5 * m_in ** 2
    assert len(np.unique(m)) == 2 and len(np.unique(v)) == 2


def test_eight_bits_follow_a_slow_decay():
    """Gradients of one element in 256 go on, the others' end: v of those loses 0.1% a step though a code is 1.6% wide and more.  After 400
    steps the mean is 0.999^400 of what it was; a step's rounding has a standard deviation below half a code (0.03 of the value there), and
    400 of them over 256 blocks of 255 average out to far less than 1%."""
    n = 256 * 256
    s = model([n], [torch.float32], 8, False)
    g = torch.full((n // 256, 256), 0.5, device="cuda")
    g[:, 0] = 1.0
    s["gs"] = [g.view(-1)]
    step(s, step=1, beta2=0.0)
    before = values(s)[1].reshape(-1, 256)[:, 1:].mean()
    g[:, 1:] = 0.0
    for t in range(2, 402):
        step(s, step=t, beta2=0.999)
    after = values(s)[1].reshape(-1, 256)[:, 1:].mean()
    assert abs(after / before - 0.999 ** 400) <= 0.01


def test_the_same_bits_again():
    a, b = model(SIZES, [torch.float32], 8, False), model(SIZES, [torch.float32], 8, False)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for t in (1, 2):
        step(a, step=t)
        with torch.cuda.stream(side):
            step(b, step=t)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a["ws"], b["ws"])) and torch.equal(a["m"], b["m"]) and torch.equal(a["v"], b["v"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [256, 256 * 37, 256 * 5000])
def test_unpack(n, dtype):
    m = torch.randint(-127, 128, (n,), device="cuda").to(torch.int8)
    v = torch.randint(0, 256, (n,), device="cuda").to(torch.uint8)
    scales = torch.rand(n // 256, 2, device="cuda")
    out = torch.full((n,), float("nan"), dtype=dtype, device="cuda"), torch.full((n,), float("nan"), dtype=dtype, device="cuda")
    gas.gas_adamw_unpack(m, v, scales, *out)
    want = R.decode(m.cpu().numpy(), v.cpu().numpy(), scales.cpu().numpy())
    for got, w in zip(out, want):
        assert (np.abs(got.double().cpu().numpy() - w) <= (6 * R.EPS32 + (R.EPS16 if dtype == torch.bfloat16 else 0)) * np.abs(w)).all()
    gas.gas_adamw_unpack(m[:0], v[:0], scales[:0], out[0][:0], out[1][:0])


@pytest.mark.parametrize("sizes", [[], [0], [1], [3, 0, 5], [16384], [16385, 1, 40_000], [32_768], [32_769, 65_536], [(911 * i) % 20_000 for i in range(260)], [5_000_001], [12] * 700])
@pytest.mark.parametrize("offset", [0, 1])
def test_squared_norm(sizes, offset):
    gen = torch.Generator().manual_seed(3)
    xs = [torch.randn(n + offset, generator=gen).cuda()[offset:] for n in sizes]
    out = torch.full((1,), float("nan"), device="cuda")
    gas.gas_sq_norms(xs, out)
    want = sum(x.double().square().sum().item() for x in xs)
    assert abs(out.item() - want) <= 1.01 * R.EPS32 * want               # one rounding of a 64-bit sum
    first = out.clone()
    gas.gas_sq_norms(xs, out)
    assert torch.equal(first, out)


def test_refusals():
    s = model([300, 20], [torch.float32], 8, False)
    step(s, step=1)
    for kw, said in ((dict(step=0), "step=0"), (dict(beta1=1.0), "beta1"), (dict(beta2=-0.1), "beta2"), (dict(eps=0.0), "eps"),
                     (dict(sq_norm=torch.zeros(1, device="cuda"), max_norm=0.0, step=1), "max_norm")):
        with pytest.raises(gas.GasError, match=said):
            step(s, **kw)
    with pytest.raises(gas.GasError, match="512 elements, 768"):
        gas.gas_adamw_steps(s["ws"], s["gs"], s["m"][:512], s["v"][:512], 0.1, 1, scales=s["scales"])
    for bad in (dict(dws=s["gs"][:1]), dict(dws=[s["gs"][1], s["gs"][0]]), dict(scales=None), dict(weight_decay=[0.1]), dict(v=s["v"][:512]),
                dict(dws=[g.bfloat16() for g in s["gs"]]), dict(master=torch.zeros(3, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            gas.gas_adamw_steps(**{**dict(ws=s["ws"], dws=s["gs"], m=s["m"], v=s["v"], lr=0.1, step=1, scales=s["scales"]), **bad})
    with pytest.raises((ValueError, TypeError)):
        gas.gas_adamw_steps([s["ws"][0][::2]], [s["gs"][0][:150].clone()], s["m"], s["v"], 0.1, 1, scales=s["scales"])
    with pytest.raises(TypeError):
        gas.gas_sq_norms([s["gs"][0].double()], torch.zeros(1, device="cuda"))
    with pytest.raises(TypeError):
        gas.gas_sq_norms([s["gs"][0].bfloat16()], torch.zeros(1, device="cuda"))
    with pytest.raises(gas.GasError, match="workspace"):
        gas.gas_sq_norms(s["gs"], torch.zeros(1, device="cuda"), workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(gas.GasError, match="n=300"):
        z = torch.zeros(300, device="cuda")
        gas.gas_adamw_unpack(torch.zeros(300, dtype=torch.int8, device="cuda"), torch.zeros(300, dtype=torch.uint8, device="cuda"), z, z, z.clone())
    gas.gas_adamw_steps([], [], s["m"], s["v"], 0.1, 1, scales=s["scales"])
