"""Workspaces of an output layer over many classes: as large as the call needs (no GPU here)."""
import pytest
import torch

import paper_2106_05609_amd as gas

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
MB = 1 << 20


def up(v, to):
    return (v + to - 1) // to * to


@pytest.mark.parametrize("n, f, c", [(1, 16, 40), (1, 64, 500), (1, 2048, 500), (8, 256, 29_360), (3, 512, 188_933), (1, 512, 4_000_000), (8, 64, 1000), (40, 64, 1000),
                                     (64, 512, 50_021), (100, 64, 1500), (512, 64, 4001), (600, 300, 3000)])
@pytest.mark.parametrize("dtype", list(DT))
def test_gradients_of_few_rows_or_classes(n, f, c, dtype):
    """X's planes for 256 rows at a time, W's for more than 64; the bias; G's planes and logits, up to 64 rows more; targets and statistics; parts of the sums: up to
    32 times GX, 32 rows at a time, and GW in fp32; of up to 64 rows' GX two for every unit or one for 128 classes; of up to eight rows' GW none."""
    planes, cp, fp = (3 if dtype == "f32" else 1), up(c, 256), up(f, 64)
    rows = n if n <= 8 else up(n, 64)
    need = 2 * planes * (up(n, 256) * fp + rows * cp + (f * up(c, 64) if n > 64 else 0)) + 4 * cp * (1 + up(n, 64) // 64) + 4 * rows * cp + 48 * up(n, 256)
    need += 16 * up(n, 16) * (cp // 256)
    need += 34 * MB if f >= 256 and n > 8 or f >= 1024 else 0
    gx = 4 * fp * max(up(rows, 32) * min(32, cp // 128), rows * min(512, cp // 128) if n <= 64 else 0)
    gw = 4 * f * cp * min(32, up(n, 256) // 128) if n > 8 else 0
    got = gas.gas_linear_xent_bwd_workspace(n, f, c, DT[dtype])
    assert got <= need + gx + gw + 8192
    assert gas.gas_linear_xent_workspace(n, f, c, DT[dtype]) <= need + 8192


@pytest.mark.parametrize("dtype", list(DT))
def test_small_calls(dtype):
    assert gas.gas_linear_xent_bwd_workspace(1, 64, 500, DT[dtype]) < MB
    assert gas.gas_linear_xent_bwd_workspace(8, 256, 29_360, DT[dtype]) < 8 * MB
    assert gas.gas_linear_distill_bwd_workspace(512, 64, 4001, DT[dtype], 16) < 32 * MB
    # a row of four million logits of 4 bytes
    assert gas.gas_linear_xent_bwd_workspace(1, 512, 4_000_000, DT[dtype]) < 80 * MB
    assert gas.gas_linear_xent_workspace(1, 512, 4_000_000, DT[dtype]) < 40 * MB


def test_workspaces_grow_with_the_call():
    """Of any more rows, inputs or classes no less, but for where another kind of tile begins."""
    sizes = lambda n, f, c: gas.gas_linear_xent_bwd_workspace(n, f, c, torch.float32)
    for f, c in ((64, 500), (300, 5000), (1100, 20_000)):
        assert sizes(1, f, c) <= sizes(5, f, c) <= sizes(8, f, c)
        assert sizes(10, f, c) <= sizes(64, f, c)
        assert sizes(65, f, c) <= sizes(200, f, c) <= sizes(2000, f, c) <= sizes(20_000, f, c)


@pytest.mark.parametrize("dtype", list(DT))
def test_top_logits_of_few_rows(dtype):
    """All logits of up to eight rows, their numbers' lists (8 bytes, two of them, k of every 2,048), a bit for each; nothing of sums that are not split."""
    for n, f, c, k in ((1, 256, 100_003, 10), (8, 256, 2000, 10), (8, 300, 700, 128)):
        assert gas.gas_linear_top_workspace(n, f, c, DT[dtype], k) <= n * (up(c, 256) * 33 // 8 + 16 * k * up(c, 2048) // 2048) + 64 * up(c, 256) // 256 + 4096
