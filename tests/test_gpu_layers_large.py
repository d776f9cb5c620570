"""The layers whose rows choose their matrices at sizes that take the kernels, tiles and launches of large calls, and the accuracy
that small results show: against their float64 definition (oracle/layers_oracle.py), or exactly where every sum is exact.
Tolerances as in test_gpu_layers.py, whose helpers this file uses."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layers_oracle as lo
from paper_2212_05231_amd import binding as nb
from test_gpu_layers import MARK, TYPES, check, empty, f64, nan_to, on_device, rows, split_rows

pytestmark = pytest.mark.gpu


# ---- more workgroups than one launch can have ------------------------------------------------------------------------------------

def test_forward_of_more_workgroups_than_a_launch_has():
    """2049 matrices of 8 to 65536 with a row each: 2049 * 4096 workgroups of 512 threads, 2^32 threads and 2 million more.  Every sum of
    8 products is checked against fp32 (8 additions) and one rounding to bf16."""
    groups, inner, outer = 2049, 8, 65536
    gen = torch.Generator(device="cuda").manual_seed(1)
    W = torch.randint(-8, 9, (groups, outer, inner), generator=gen, device="cuda", dtype=torch.int8).bfloat16()
    x = torch.randint(-8, 9, (groups, inner), generator=gen, device="cuda", dtype=torch.int8).bfloat16()
    y = torch.full((groups, outer), MARK, dtype=torch.bfloat16, device="cuda")
    nb.grouped_fwd(nb.make_layer("bf16", groups, inner, outer), x, W, on_device(list(range(groups + 1))), y)
    for g in range(0, groups, 128):
        want = (W[g:g + 128].float() * x[g:g + 128, None].float()).sum(2)            # whole numbers: exact
        assert torch.equal(y[g:g + 128], want.bfloat16()), g


def test_gradients_of_more_workgroups_than_a_launch_has():
    """32769 matrices of 65536 to 1 with a row each: 32769 * 1024 tiles for dx and 32770 * 512 for dW.  Every result is one product."""
    groups, inner = 32769, 65536
    gen = torch.Generator(device="cuda").manual_seed(2)
    W = torch.randint(-127, 128, (groups, 1, inner), generator=gen, device="cuda", dtype=torch.int8).bfloat16()
    x = torch.randint(-127, 128, (groups, inner), generator=gen, device="cuda", dtype=torch.int8).bfloat16()
    dy = torch.randint(-127, 128, (groups, 1), generator=gen, device="cuda", dtype=torch.int8).bfloat16()
    layer = nb.make_layer("bf16", groups, inner, 1)
    dx = torch.full((groups, inner), MARK, dtype=torch.bfloat16, device="cuda")
    dW = torch.full((groups, 1, inner), MARK, device="cuda")
    need = nb.grouped_workspace_bytes(layer, groups)
    nb.grouped_bwd(layer, x, W, on_device(list(range(groups + 1))), dy, dx, dW, torch.zeros(max(need // 4, 4), device="cuda"))
    for g in range(0, groups, 1024):
        part = slice(g, g + 1024)
        assert torch.equal(dx[part], (W[part, 0].float() * dy[part].float()).bfloat16()), g
        assert torch.equal(dW[part, 0], x[part].float() * dy[part].float()), g
