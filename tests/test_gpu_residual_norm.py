"""gas_residual_norm and its backward against their definitions in 64 bits (tests/residual_reference.py).

Errors are measured in units of half a last place of float32 times the magnitude a result is summed from (and, for stored bf16, half a
last place of bf16 of the value).  A row's sums take at most F / 64 + 7 additions one after another and a few products and a root, the
sums over the rows n / 64 + 64; `UNITS` allows for a handful of such sums behind one another."""
import itertools

import pytest
import torch

import paper_2106_05609_amd as gas
from tests import residual_reference as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = [(1, 1), (3, 2), (2, 3), (5, 7), (4, 8), (67, 8), (700, 5), (260, 9), (513, 12), (301, 16), (1030, 4), (130, 24), (33, 31), (130, 47), (1, 64), (257, 64), (66, 65), (63, 100), (129, 128), (1000, 200), (1, 256),
         (300, 256), (31, 257), (40, 512), (9, 520), (21, 1000), (19, 1433), (7, 2048), (6, 2049), (5, 4100), (3, 8200), (2, 16384), (2, 16390)]


def units(f):
    return 96 + f / 8


def make(n, f, dtype, gate, bias=True, seed=0, shift=0.0, ld=None, off=0):
    """Inputs on the GPU; ld, off: row stride and first element of every matrix."""
    gen = torch.Generator().manual_seed(seed + 1000 * n + f)
    r = lambda *s: torch.randn(*s, generator=gen)

    def mat(cols, scale=1.0, plus=0.0):
        step = cols if ld is None else ld
        flat = torch.zeros(off + max(1, n) * step, dtype=DT[dtype], device="cuda")
        m = torch.as_strided(flat, (n, cols), (step, 1), off)
        m.copy_((r(n, cols) * scale + plus).to(DT[dtype]))
        return m
    vec = lambda around: (around + 0.3 * r(f)).cuda()
    c = dict(x=mat(f, 1.5, shift), a=mat(f, 0.7, shift), t=None if gate == 0 else mat(f if gate == 2 else 1), p=vec(1.0), p_bias=vec(0.0) if bias else None,
             s=vec(0.5), q=vec(1.0), q_bias=vec(0.0) if bias else None, alpha=0.7, eps=1e-5)
    return c, mat


def wide(c):
    return {k: v.double().cpu() if torch.is_tensor(v) else v for k, v in c.items()}


def check(got, want, mag, dtype, k, what):
    got = got.double().cpu()
    allowed = R.EPS32 * k * mag + (R.EPS16 * want.abs() if dtype == "bf16" else 0)
    worst = ((got - want).abs() / (allowed + 1e-30)).max().item() if got.numel() else 0.0
    assert worst <= 1.0, (what, worst)


def forward_mag(d, h, u, stats, post, pre):
    """Magnitudes of h and u, row by row: what a relative error of the row's statistics can move."""
    one = lambda v: 1.0 if v is None else v.abs()
    am = (d["a"].abs() + stats[:, 0:1].abs()) * stats[:, 1:2]
    am = am + am.amax(1, keepdim=True) * (post != R.NONE)
    y = am * one(d["p"]) + (0.0 if d["p_bias"] is None else d["p_bias"].abs())
    hm = d["x"].abs() + abs(d["alpha"]) * one(d["s"]) * y
    top = hm.amax(1, keepdim=True) if pre != R.NONE else 0.0
    um = (hm + stats[:, 2:3].abs() + top) * stats[:, 3:4] * one(d["q"]) + (0.0 if d["q_bias"] is None else d["q_bias"].abs())
    return hm, um


def run_forward(c, post, pre, h=True, u=True, stats=True, **kw):
    empty = lambda: torch.full_like(c["x"], float("nan"))
    out = dict(h=kw.pop("h_out", empty()) if h else None, u=kw.pop("u_out", empty()) if u else None,
               stats=torch.full((c["x"].shape[0], 4), float("nan"), device="cuda") if stats else None)
    gas.gas_residual_norm(c["x"], h=out["h"], u=out["u"], stats=out["stats"], post=post, pre=pre, **{k: v for k, v in c.items() if k != "x"}, **kw)
    return out


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("n,f", SIZES)
def test_forward(n, f, dtype):
    for (post, pre), gate in zip([(2, 2), (1, 1), (0, 2), (2, 0), (1, 2)], [2, 1, 0, 2, 2]):
        c, _ = make(n, f, dtype, gate, bias=post == 2, shift=0.5 * post)
        out = run_forward(c, post, pre)
        h, u, stats = R.forward(post=post, pre=pre, **wide(c))
        hm, um = forward_mag(wide(c), h, u, stats, post, pre)
        check(out["h"], h, hm, dtype, units(f), ("h", post, pre, gate))
        check(out["u"], u, um, dtype, units(f), ("u", post, pre, gate))
        check(out["stats"][:, 1::2], stats[:, 1::2], stats[:, 1::2] * (1 + hm.amax(1, keepdim=True) * stats[:, 3:4]), "f32", units(f), "deviations")


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("n,f", SIZES)
def test_backward(n, f, dtype):
    for (post, pre), gate in zip([(2, 2), (1, 1), (0, 2), (2, 0), (1, 2)], [2, 1, 0, 2, 1]):
        c, mat = make(n, f, dtype, gate, bias=post == 2, shift=0.25 * post)
        fwd = run_forward(c, post, pre)
        gh, gu = mat(f), mat(f)
        got = run_backward(c, fwd, gh, gu, post, pre)
        compare_backward(c, fwd, gh, gu, post, pre, got, dtype)


def run_backward(c, fwd, gh, gu, post, pre, into=None, **only):
    x = c["x"]
    new = lambda: torch.full(x.shape, float("nan"), dtype=x.dtype, device="cuda")
    out = dict(gx=new(), ga=new(), gt=None if c["t"] is None else torch.full(c["t"].shape, float("nan"), dtype=x.dtype, device="cuda"))
    for k in ("gp", "gp_bias", "gs", "gq", "gq_bias"):
        out[k] = torch.full((x.shape[1],), float("nan"), device="cuda")
    out.update(into or {})
    out.update(only)
    gas.gas_residual_norm_bwd(gh, gu, fwd["h"], fwd["stats"], a=c["a"], t=c["t"], post=post, p=c["p"], p_bias=c["p_bias"], s=c["s"], alpha=c["alpha"],
                              pre=pre, q=c["q"], **out)
    return {k: v for k, v in out.items() if v is not None}


def compare_backward(c, fwd, gh, gu, post, pre, got, dtype):
    d = wide(c)
    n, f = c["x"].shape
    w64 = lambda v: None if v is None else v.double().cpu()
    want, mag = R.backward(w64(gh), w64(gu), w64(fwd["h"]), w64(fwd["stats"]), d["a"], d["t"], 0 if d["t"] is None else d["t"].shape[1], post, d["p"],
                           d["p_bias"], d["s"], d["alpha"], pre, d["q"])
    for k, v in got.items():
        rows = k in ("gx", "ga", "gt")
        check(v, want[k], mag[k], dtype if rows else "f32", units(f) + (0 if rows else 64 + n / 16), (k, post, pre))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("n,f,ld,off", [(37, 64, 67, 1), (21, 100, 104, 3), (18, 256, 257, 5), (9, 1433, 1440, 2), (5, 1, 3, 1), (11, 7, 9, 1), (4, 5000, 5001, 1)])
def test_strides_and_alignment(n, f, ld, off, dtype):
    for gate in (1, 2):
        c, mat = make(n, f, dtype, gate, ld=ld, off=off)
        h, u, gx = mat(f), mat(f), mat(f)
        between = torch.as_strided(h, (n, ld - f), (ld, 1), h.storage_offset() + f) if n > 1 else None
        between = between[:-1]                                       # the last row's may lie past the end
        between.fill_(7.0)
        fwd = run_forward(c, 2, 2, h_out=h, u_out=u)
        d = wide(c)
        hw, uw, stats = R.forward(post=2, pre=2, **d)
        hm, um = forward_mag(d, hw, uw, stats, 2, 2)
        check(h, hw, hm, dtype, units(f), "h")
        check(u, uw, um, dtype, units(f), "u")
        gh, gu = mat(f), mat(f)
        got = run_backward(c, fwd, gh, gu, 2, 2, into=dict(gx=gx))
        compare_backward(c, fwd, gh, gu, 2, 2, got, dtype)
        assert (between == 7.0).all()                                # what lies between the rows is left alone


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("f", [8, 47, 64, 256, 1433, 5000])
def test_in_place(f, dtype):
    n = 70
    for gate in (1, 2):
        c, mat = make(n, f, dtype, gate)
        fwd = run_forward(c, 2, 1)
        d = dict(c, x=c["x"].clone(), a=c["a"].clone())
        out = run_forward(d, 2, 1, h_out=d["x"], u_out=d["a"])
        assert torch.equal(out["h"], fwd["h"]) and torch.equal(out["u"], fwd["u"]) and torch.equal(out["stats"], fwd["stats"])
        gh, gu = mat(f), mat(f)
        got = run_backward(c, fwd, gh, gu, 2, 1)
        d, g = dict(c, a=c["a"].clone(), t=c["t"].clone()), gh.clone()
        again = run_backward(d, fwd, g, gu, 2, 1, into=dict(gx=g, ga=d["a"], gt=d["t"]))
        for k in got:
            assert torch.equal(got[k], again[k]), k


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("f", [47, 257, 1433, 1541, 3999])
def test_in_place_without_norms(f, dtype):
    """Nothing that the row's wavefronts would wait for lies between reading and storing; the last 16 bytes of a row of odd width are read twice."""
    n = 3000
    c, mat = make(n, f, dtype, 2)
    fwd = run_forward(c, 0, 0)
    d = dict(c, x=c["x"].clone(), a=c["a"].clone())
    out = run_forward(d, 0, 0, h_out=d["x"], u_out=d["a"])
    assert torch.equal(out["h"], fwd["h"]) and torch.equal(out["u"], fwd["u"])
    gh, gu = mat(f), mat(f)
    got = run_backward(c, fwd, gh, gu, 0, 0)
    d, g = dict(c, a=c["a"].clone(), t=c["t"].clone()), gh.clone()
    again = run_backward(d, fwd, g, gu, 0, 0, into=dict(gx=g, ga=d["a"], gt=d["t"]))
    for k in got:
        assert torch.equal(got[k], again[k]), k


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("n,f", [(1, 64), (300, 64), (77, 47), (40, 1433), (3, 5000)])
def test_only_some_outputs(n, f, dtype):
    c, mat = make(n, f, dtype, 2)
    both = run_forward(c, 2, 2)
    assert torch.equal(run_forward(c, 2, 2, u=False, stats=False)["h"], both["h"])
    assert torch.equal(run_forward(c, 2, 2, h=False, stats=False)["u"], both["u"])
    bare = {"x": c["x"], "a": None, "t": None, "p": None, "p_bias": None, "s": None, "q": c["q"], "q_bias": c["q_bias"], "alpha": 1.0, "eps": 1e-5}
    out = run_forward(bare, 0, 2)
    assert torch.equal(out["h"], c["x"])
    d = wide(c)
    h, u, stats = R.forward(d["x"], None, None, 0, None, None, None, 1.0, 2, d["q"], d["q_bias"], 1e-5)
    check(out["u"], u, ((d["x"].abs() + d["x"].abs().amax(1, keepdim=True) * 2) * stats[:, 3:4] * d["q"].abs() + d["q_bias"].abs()), dtype, units(f), "u")
    gh, gu = mat(f), mat(f)
    full = run_backward(c, both, gh, gu, 2, 2)
    for keep in ("gx", "ga", "gt", "gp", "gq_bias"):
        none = {k: None for k in full if k != keep}
        assert torch.equal(run_backward(c, both, gh, gu, 2, 2, **none)[keep], full[keep]), keep
    # no gradient at the stream, none at the normed rows, no block
    got = run_backward(c, both, None, gu, 2, 2)
    compare_backward(c, both, None, gu, 2, 2, got, dtype)
    got = run_backward(c, both, gh, None, 2, 2, gq=None, gq_bias=None)
    compare_backward(c, both, gh, None, 2, 2, got, dtype)
    nothing = dict(c, a=None, t=None, p=None, p_bias=None, s=None)
    got = run_backward(nothing, both, gh, gu, 0, 2, ga=None, gt=None, gp=None, gp_bias=None, gs=None)
    assert torch.equal(got["gx"], full["gx"]) and torch.equal(got["gq"], full["gq"])


@pytest.mark.parametrize("f", [16, 47, 256, 1433, 5000])
def test_push(f):
    for dtype in DT:
        c, _ = make(33, f, dtype, 2)
        want = run_forward(c, 2, 2)
        hist = torch.full((101, f), 3.0, dtype=DT[dtype], device="cuda")
        idx = torch.randperm(101, device="cuda")[:33].to(torch.int32)
        out = run_forward(c, 2, 2, idx=idx, hist=hist)
        assert torch.equal(out["u"], want["u"]) and torch.equal(hist[idx.long()], want["u"])
        rest = torch.ones(101, dtype=torch.bool, device="cuda")
        rest[idx.long()] = False
        assert (hist[rest] == 3.0).all()
        alone = torch.zeros_like(hist)
        run_forward(c, 2, 2, h=False, u=False, stats=False, idx=idx, hist=alone)
        assert torch.equal(alone[idx.long()], want["u"])


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("f", [7, 64, 256, 1433, 5000])
def test_rows_with_infinities_constant_rows_and_shut_gates(f, dtype):
    n = 40
    c, mat = make(n, f, dtype, 2)
    c["x"][3] = 2.0
    c["a"][3] = 0.0                                    # a constant row: no deviation, u = q_bias
    c["s"][:] = 0.5
    c["p_bias"][:] = 0.0
    c["a"][5], c["x"][5] = 0.0, 0.0
    clean = run_forward(c, 2, 2)
    for k in ("h", "u", "stats"):
        assert torch.isfinite(clean[k]).all(), k
    assert torch.equal(clean["u"][3], c["q_bias"].to(DT[dtype])) and torch.equal(clean["h"][3], c["x"][3])
    gh, gu = mat(f), mat(f)
    back = run_backward(c, clean, gh, gu, 2, 2)
    assert all(torch.isfinite(v).all() for v in back.values())
    # gates that are shut or open for good: logits of the type's lowest and largest value, and infinite ones
    shut = dict(c, t=c["t"].clone())
    low = torch.finfo(DT[dtype]).min
    shut["t"][0], shut["t"][1], shut["t"][2], shut["t"][4] = low, float("-inf"), -low, float("inf")
    out = run_forward(shut, 2, 2)
    assert torch.equal(out["h"][0], c["x"][0]) and torch.equal(out["h"][1], c["x"][1])
    got = run_backward(shut, out, gh, gu, 2, 2)
    assert all(torch.isfinite(v).all() for v in got.values())
    assert (got["gt"][[0, 1, 2, 4]] == 0).all() and (got["ga"][:2] == 0).all()
    # an infinity or a NaN of a row stays in the row
    for where, value in (("x", float("inf")), ("a", float("nan")), ("x", float("nan")), ("a", float("-inf"))):
        bad = dict(c, **{where: c[where].clone()})
        bad[where][7, f // 2] = value
        out = run_forward(bad, 2, 2)
        assert not torch.isfinite(out["u"][7]).all()
        rest = [i for i in range(n) if i != 7]
        assert torch.equal(out["h"][rest], clean["h"][rest]) and torch.equal(out["u"][rest], clean["u"][rest])
        got = run_backward(bad, out, gh, gu, 2, 2)
        for k in ("gx", "ga", "gt"):
            assert torch.equal(got[k][rest], back[k][rest]), k


@pytest.mark.parametrize("f", [64, 256, 1433])
def test_gradients_by_differences(f):
    """L = <gh, h> + <gu, u> along a direction: (L(+e) - L(-e)) / 2 e, outputs of float32 (half a last place of about 4 each), sums in
    64 bits: n f errors at random are 2 * 4 * 2^-24 * sqrt(n f) / 2 e; the third derivative's share is e^2 times some 10 |slope scale|."""
    n, e = 24, 1e-2
    c, mat = make(n, f, "f32", 2)
    gh, gu = mat(f), mat(f)
    fwd = run_forward(c, 2, 1)
    got = run_backward(c, fwd, gh, gu, 2, 1)

    def loss(**kw):
        out = run_forward(dict(c, **kw), 2, 1)
        return (out["h"].double() * gh.double()).sum() + (out["u"].double() * gu.double()).sum()
    for k in ("x", "a", "t", "p", "p_bias", "s", "q", "q_bias"):
        d = torch.randn_like(c[k])
        slope = (loss(**{k: c[k] + e * d}) - loss(**{k: c[k] - e * d})) / (2 * e)
        want = (got["g" + k].double() * d.double()).sum()
        scale = got["g" + k].double().norm() * d.double().norm() / d.numel() ** 0.5
        assert abs(slope - want) <= 40 * (n * f) ** 0.5 * R.EPS32 / e * 4 + 30 * e * e * scale * 4, (k, slope.item(), want.item())


def test_the_same_bits_again_and_on_another_stream():
    for n, f in ((5000, 256), (700, 1433), (333, 47)):
        c, mat = make(n, f, "bf16", 2)
        gh, gu = mat(f), mat(f)
        fwd = run_forward(c, 2, 2)
        got = run_backward(c, fwd, gh, gu, 2, 2)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            fwd2 = run_forward(c, 2, 2)
            got2 = run_backward(c, fwd2, gh, gu, 2, 2)
        side.synchronize()
        assert all(torch.equal(fwd[k], fwd2[k]) for k in fwd) and all(torch.equal(got[k], got2[k]) for k in got)


def test_many_rows():
    """Sums over more rows than the grid holds at once, and offsets that pass 32 bits (rows of 1,000 from 2.3 million elements apart)."""
    c, mat = make(70_001, 64, "f32", 2)
    fwd = run_forward(c, 2, 2)
    gh, gu = mat(64), mat(64)
    compare_backward(c, fwd, gh, gu, 2, 2, run_backward(c, fwd, gh, gu, 2, 2), "f32")
    n, f, ld = 2000, 1000, 2_300_001
    far = torch.as_strided(torch.zeros(n * ld, dtype=torch.bfloat16, device="cuda"), (n, f), (ld, 1))
    far.copy_(torch.randn(n, f, device="cuda").bfloat16())
    near = dict(x=far.contiguous(), a=None, t=None, p=None, p_bias=None, s=None, q=None, q_bias=None, alpha=1.0, eps=1e-5)
    want = run_forward(near, 0, 2)
    gas.gas_residual_norm(far, h=far, u=(u := torch.empty_like(near["x"])), pre=2)
    assert torch.equal(u, want["u"]) and torch.equal(far, near["x"])


@pytest.mark.parametrize("n,f,dtype", [(600_001, 8, "f32"), (530_003, 64, "f32"), (1_100_003, 8, "bf16"), (300_007, 40, "bf16"), (131_101, 505, "bf16"), (65_601, 700, "f32")])
def test_sums_over_thousands_of_workgroups(n, f, dtype):
    """So many rows that the workgroups' sums are added up in two launches."""
    c, mat = make(n, f, dtype, 2)
    fwd = run_forward(c, 2, 2)
    gh, gu = mat(f), mat(f)
    compare_backward(c, fwd, gh, gu, 2, 2, run_backward(c, fwd, gh, gu, 2, 2), dtype)


def test_no_rows():
    c, mat = make(0, 64, "f32", 2)
    fwd = run_forward(c, 2, 2)
    got = run_backward(c, fwd, mat(64), mat(64), 2, 2)
    for k in ("gp", "gp_bias", "gs", "gq", "gq_bias"):
        assert (got[k] == 0).all()


def test_refusals():
    c, mat = make(6, 64, "f32", 2)
    h, u = torch.empty_like(c["x"]), torch.empty_like(c["x"])
    call = lambda **kw: gas.gas_residual_norm(**{**dict(x=c["x"], h=h, u=u, a=c["a"], t=c["t"], post=2, p=c["p"], pre=2, q=c["q"]), **kw})
    call()
    flat = torch.zeros(6 * 64 + 8, device="cuda")
    shifted = torch.as_strided(flat, (6, 64), (64, 1), 4)
    for kw, said in ((dict(post=3), "unknown norm"), (dict(pre=-1), "unknown norm"), (dict(eps=0.0), "eps"), (dict(a=None), "gate without"),
                     (dict(h=None, u=None), "null"), (dict(u=h), "share memory"), (dict(x=flat[:384].view(6, 64), h=shifted), "lies in an input"),
                     (dict(eps=float("nan")), "eps"), (dict(t=torch.zeros(6, 3, device="cuda")), "3 gates"),
                     (dict(idx=torch.arange(6, dtype=torch.int32, device="cuda"), hist=torch.zeros(5, 64, device="cuda")), "history"),
                     (dict(idx=torch.arange(6, dtype=torch.int32, device="cuda"), hist=c["a"]), "history table lies")):
        with pytest.raises(gas.GasError, match=said):
            call(**kw)
    for kw in (dict(h=h[:5]), dict(u=u.bfloat16()), dict(p=c["p"][:63]), dict(a=c["a"][:, :63]), dict(stats=torch.zeros(6, 3, device="cuda")),
               dict(idx=torch.arange(6, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(TypeError):
        call(p=c["p"].double())
    fwd = run_forward(c, 2, 2)
    gh, gu, gx = mat(64), mat(64), mat(64)
    back = lambda **kw: gas.gas_residual_norm_bwd(**{**dict(gh=gh, gu=gu, h=fwd["h"], stats=fwd["stats"], gx=gx, a=c["a"], t=c["t"], post=2, pre=2), **kw})
    back()
    for kw, said in ((dict(gx=None), "null"), (dict(h=None), "without the rows"), (dict(stats=None), "without statistics"),
                     (dict(a=None, t=None, ga=gx), "without the block"), (dict(gu=None, gq=c["q"].clone()), "without the gradient"),
                     (dict(t=None, gt=torch.zeros(6, 64, device="cuda")), "do not match"), (dict(ga=gx), "share memory"), (dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), "workspace")):
        with pytest.raises((gas.GasError, ValueError), match=said):
            back(**kw)
    with pytest.raises(ValueError):
        back(gh=None, gu=None, gx=None)
    # columns of one matrix are apart
    wide_ = torch.zeros(6, 128, device="cuda")
    call(x=wide_[:, :64], h=wide_[:, 64:])
