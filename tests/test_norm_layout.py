"""How rows lie in the lanes of the norms' kernels (paper_2106_05609_amd/csrc/norm_layout.h): csrc/norm_check.cpp under the address and
undefined-behaviour sanitizers.  Host code only; no GPU is involved."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2106_05609_amd", "csrc")


@pytest.fixture(scope="module")
def checker(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("norm") / "norm_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-o", exe,
                           os.path.join(CSRC, "norm_check.cpp")])
    return exe


def run(*cmd):
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1", UBSAN_OPTIONS="halt_on_error=1")
    res = subprocess.run(cmd, env=env, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-4000:]
    assert " 0 failures" in res.stdout


def test_pieces_lie_in_their_rows(checker):
    run(checker, "pieces")


def test_offsets_in_32_bits(checker):
    run(checker, "offsets")


def test_workgroups_for_any_number_of_rows(checker):
    run(checker, "rows")


def test_workspace_of_the_backward_pass_is_bounded():
    """At most 1 MB for every column while rows are whole in registers, however many there are."""
    from paper_2106_05609_amd import binding as B
    for f in (1, 8, 47, 64, 256, 400, 768, 1433, 4096):
        for n in (1, 600_000, 3_125_002, 24_700_000, 111_059_956, 1 << 33):
            assert B.gas_residual_norm_bwd_workspace(n, f) <= (1 << 20) * f, (n, f)


def test_workspace_of_either_type():
    import torch
    from paper_2106_05609_amd import binding as B
    for f in (1, 7, 64, 256, 600, 1433, 5000, 9000):
        last = {}
        for n in [*range(0, 3000, 13), 50_000, 262_143, 600_000, 3_125_002, 111_059_956]:
            both = [B.gas_residual_norm_bwd_workspace(n, f, dt) for dt in (torch.float32, torch.bfloat16)]
            assert max(both) == B.gas_residual_norm_bwd_workspace(n, f)
            for dt, need in enumerate(both):
                assert need >= last.get(dt, 0)
                last[dt] = need
    assert B.gas_residual_norm_bwd_workspace(200_000, 600, torch.bfloat16) == 256 * 5 * 600 * 4
    with pytest.raises(TypeError):
        B.gas_residual_norm_bwd_workspace(1, 1, torch.float16)
