"""csrc/marshal.cpp: lists of tensors and of vectors against the Python functions they stand in for, and what they leave to those."""
import array

import pytest
import torch

from paper_2106_05609_amd import binding as B

L = B._calls()
from paper_2106_05609_amd import _marshal as M      # noqa: E402


class Sub(torch.Tensor):
    pass


base = torch.arange(60, dtype=torch.float32).view(6, 10)


def test_lists_of_tensors():
    ts = [base, base.bfloat16(), base[0], base[:0], torch.nn.Parameter(base.clone()), base[1:4]]
    assert M.tensors(ts) == B._tensors_any(ts) == M.tensors(tuple(ts))
    assert M.tensors([]) == (b"", b"", b"") == B._tensors_any([])
    for left in (base.t(), base.double(), base.as_subclass(Sub), None, 3):
        assert M.tensors([base, left]) is None
    with pytest.raises(TypeError):
        M.tensors(3)
    with pytest.raises(ValueError):
        B._tensors([base, base[:, ::2]])
    with pytest.raises(TypeError):
        B._tensors([base, base.int()])
    assert B._tensors([base.as_subclass(Sub)]) == B._tensors_any([base])


def test_numbers():
    vs = [0.1, 1, 2.5e-7, float("inf")]
    assert M.floats(vs) == B._floats_any(vs) == array.array("f", vs).tobytes()
    assert M.floats(()) == b""
    with pytest.raises(TypeError):
        M.floats(["x"])
    with pytest.raises(TypeError):
        M.floats(1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_matrices_of_one_size(dtype):
    x = base.to(dtype)
    wide = torch.zeros(6, 30, dtype=dtype)
    ts = [x, None, wide[:, 10:20], x[:6]]
    assert M.alike(x, *ts) == B._alike_any("", x, *ts) == B._alike("", x, *ts)
    assert M.alike(x) == (6, 10, B._dt(x))
    assert M.alike(x[:0], x[:0], None) == B._alike_any("", x[:0], x[:0], None)
    for other in (x[:5], wide, x.to(torch.float16), base.t(), base.to(torch.bfloat16 if dtype == torch.float32 else torch.float32)):
        assert M.alike(x, x, other) is None
        with pytest.raises(ValueError):
            B._alike("who", x, x, other)
    assert M.alike(3) is None and M.alike(x.as_subclass(Sub), x) is None
    assert B._alike("", x.as_subclass(Sub), x) == B._alike_any("", x, x)


def test_vectors_of_one_width():
    v = torch.zeros(10)
    assert M.vectors(10, v, None, base[0]) == B._vectors_any("", 10, v, None, base[0]) == B._vectors("", 10, v, None, base[0])
    assert M.vectors(10) == ()
    assert M.vectors(10, v.double()) is None and M.vectors(9, v) is None and M.vectors(6, base[:, 0]) is None
    with pytest.raises(ValueError, match="a vector of 10 for rows of 9"):
        B._vectors("who", 9, v)
    with pytest.raises(ValueError, match="contiguous"):
        B._vectors("who", 6, base[:, 0])
    with pytest.raises(TypeError):
        B._vectors("who", 10, v.double())
    with pytest.raises(TypeError):
        M.vectors("x", v)


def test_without_the_module(monkeypatch):
    """The calls work through the Python functions too."""
    for name in ("_tensors", "_floats", "_alike", "_vectors"):
        monkeypatch.setattr(B, name, getattr(B, name + "_any"))
    monkeypatch.setattr(B, "_stream", lambda: 0)
    x = base[:0]
    B.gas_residual_norm(x, h=x.clone(), u=x.clone(), q=torch.zeros(10), pre=B.NORM_RMS)
    B.gas_residual_norm_bwd(x, None, None, None, gx=x.clone())
    B.gas_adamw_steps([], [], torch.zeros(0), torch.zeros(0), 0.1, 1)
    with pytest.raises(ValueError, match="weight decay"):
        B.gas_adamw_steps([base], [base], torch.zeros(256), torch.zeros(256), 0.1, 1, weight_decay=[0.1, 0.2])
    assert B.gas_adamw_elements([1, 256, 257, 0]) == 256 + 256 + 512
