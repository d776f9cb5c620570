"""The layers whose rows choose their matrices at sizes that take the kernels, tiles and launches of large calls, and the accuracy
that small results show: against their float64 definition (oracle/layers_oracle.py), or exactly where every sum is exact.
Tolerances as in test_gpu_layers.py, whose helpers this file uses."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layers_oracle as lo
from paper_2212_05231_amd import binding as nb
from paper_2212_05231_amd import layers as rows_layers
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


# ---- what is left where large parts cancel ---------------------------------------------------------------------------------------------

def three_terms(v):
    """fp32 v as its bf16 rounding, that of the rest, and the rest of both."""
    hi = v.bfloat16().float()
    mid = (v - hi).bfloat16().float()
    return hi, mid, v - hi - mid


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,inner,outer", [(16, 64, 64), (300, 64, 64), (66000, 64, 64), (17000, 72, 520), (17000, 520, 72), (8400, 64, 1024), (8400, 1024, 64)])
def test_adapters_add_all_of_u_and_v(n, inner, outer, dtype):
    """Rows in which W x (backward: W^T dy) takes away the first two bf16 terms of B u (A^T v): what comes out is the third one, of at most
    7 bits.  u and v hold all 24 bits of a scale; every product and partial sum is a multiple of 2^-23 below 2: nothing is rounded."""
    gen = torch.Generator().manual_seed(n + outer)
    slots, rank, groups = 8, 8, 20
    s = 1.0 + torch.rand(slots, generator=gen) * 0.9
    hi, mid, rest = three_terms(s)
    assert (rest != 0).sum() >= 6 and rest.abs().max() <= 2.0 ** -17
    named = [g % slots for g in range(groups)]
    off = split_rows(n, groups, gen)
    scales, slot_of_row = s.cuda(), torch.zeros(n, dtype=torch.long)
    for g in range(groups):
        slot_of_row[off[g]:off[g + 1]] = named[g]
    ones = lambda width: torch.zeros(n, width).scatter_(1, 2 * slot_of_row[:, None] + torch.arange(2), 1.0).to(TYPES[dtype]).cuda()
    part = torch.stack((-hi, -mid), 1).reshape(16)                                     # what the shared matrix takes away
    A, B = torch.zeros(slots, rank, inner), torch.zeros(slots, outer, rank)
    layer = nb.make_layer(dtype, groups, inner, outer, rank=rank, adapters=slots)
    move = lambda t: t.to(TYPES[dtype]).cuda()
    # forward: u = s A x = s
    W = torch.zeros(outer, inner)
    W[:, :16] = part
    A[torch.arange(slots), 0, 2 * torch.arange(slots)] = 1.0
    B[:, :, 0] = 1.0
    assert torch.equal(move(W).float().cpu(), W)
    y, u = empty(n, outer, outer, dtype), torch.full((n, rank), MARK, device="cuda")
    nb.adapter_fwd(layer, ones(inner), move(W), move(A), move(B), scales, on_device(named), on_device(off), u, y)
    assert torch.equal(u[:, 0].cpu(), s[slot_of_row])
    assert torch.equal(y.float().cpu(), rest[slot_of_row][:, None].expand(n, outer))
    # backward: v = s B^T dy = s
    W, A, B = torch.zeros(outer, inner), torch.zeros_like(A), torch.zeros_like(B)
    W[:16] = part[:, None]
    B[torch.arange(slots), 2 * torch.arange(slots), 0] = 1.0
    A[:, 0, :] = 1.0
    dx = empty(n, inner, inner, dtype)
    workspace = torch.zeros(nb.adapter_workspace_bytes(layer, n) // 4, device="cuda")
    nb.adapter_bwd(layer, None, move(W), move(A), move(B), scales, on_device(named), on_device(off), None, ones(outer), dx, None, None, workspace)
    assert torch.equal(dx.float().cpu(), rest[slot_of_row][:, None].expand(n, inner))


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,groups,slots,inner,outer,rank", [(700, 5, 3, 136, 200, 64), (1500, 100, 30, 300, 129, 33), (900, 9, 4, 256, 64, 8)])
def test_gradients_of_adapters_take_three_terms(n, groups, slots, inner, outer, rank, dtype, packed, accumulate):
    """dA and dB of 16-bit layers are fp32 results of fp32 u and v: as near as those of an fp32 layer (two terms: 2^-17 a product)."""
    gen = torch.Generator().manual_seed(n)
    off, named = split_rows(n, groups, gen), torch.randint(0, slots, (groups,), generator=gen).tolist()
    x, dy = rows(n, inner, inner, dtype, gen), rows(n, outer, outer, dtype, gen, 0.01)
    W = (torch.randn(outer, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    A = (torch.randn(slots, rank, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    B = (torch.randn(slots, outer, rank, generator=gen) * rank ** -0.5).to(TYPES[dtype]).cuda()
    scales, u = (torch.rand(slots, generator=gen) + 0.5).cuda(), torch.randn(n, rank, generator=gen).cuda()
    q8, e8, _ = lo.pack8(f64(x), dtype)
    x64 = lo.unpack8(q8, e8, inner) if packed else f64(x)
    given = (torch.as_tensor(q8).cuda(), torch.as_tensor(e8).cuda()) if packed else x
    args = (f64(W), f64(A), f64(B), f64(scales), named, off)
    _, want_dA, want_dB = lo.adapter_backward(x64, *args, f64(u), f64(dy))
    layer = nb.make_layer(dtype, groups, inner, outer, rank=rank, adapters=slots, accumulate=bool(accumulate))
    dA, dB = (torch.randn(w.shape, generator=gen).cuda() * float(np.abs(w).mean()) for w in (want_dA, want_dB))
    start = [f64(t) if accumulate else 0.0 for t in (dA, dB)]
    workspace = torch.zeros(nb.adapter_workspace_bytes(layer, n) // 4, device="cuda")
    nb.adapter_bwd(layer, given, None, A, B, scales, on_device(named), on_device(off), u, dy, None, dA, dB, workspace)
    for got, want, s in zip((dA, dB), (want_dA, want_dB), start):
        assert np.linalg.norm(f64(got) - (want + s)) <= 2e-6 * np.linalg.norm(want)


# ---- the ends of the range of numbers ---------------------------------------------------------------------------------------------------

LARGEST = torch.finfo(torch.float32).max                     # bf16's largest number is 0.4 % smaller


@pytest.mark.parametrize("n,inner,outer", [(8, 64, 64), (200, 64, 64), (600, 100, 104), (17000, 72, 520), (66000, 64, 40)])
def test_fp32_factors_up_to_the_largest_number(n, inner, outer):
    """One of them in each factor of every product; the results are finite."""
    gen = torch.Generator().manual_seed(n)
    small = lambda *shape: torch.randn(*shape, generator=gen).clamp(-3, 3) * 1e-3
    x, dy, W = small(n, inner), small(n, outer), small(3, outer, inner)
    x[1, inner // 2], dy[n // 2, 2] = LARGEST, -LARGEST
    W[1, 1, 0], W[0, 3, 5] = -LARGEST, LARGEST * 0.998
    x, dy, W, off = x.cuda(), dy.cuda(), W.cuda(), [0, n // 3, n // 2, n]
    layer = nb.make_layer("f32", 3, inner, outer)
    y, dx, dW = empty(n, outer, outer, "f32"), empty(n, inner, inner, "f32"), torch.zeros(3, outer, inner, device="cuda")
    nb.grouped_fwd(layer, x, W, on_device(off), y)
    q, e = torch.zeros(n, (inner + 31) // 32 * 32, dtype=torch.int8, device="cuda"), torch.zeros(n, (inner + 31) // 32, dtype=torch.uint8, device="cuda")
    nb.pack8(x, q, e)
    sizes = [np.abs(f64(t)) for t in (x, W, dy)]
    check(y, lo.grouped_forward(f64(x), f64(W), off), lo.grouped_forward(sizes[0], sizes[1], off), "f32", inner, "y")
    for given, kept in ((x, f64(x)), ((q, e), lo.unpack8(q.cpu().numpy(), e.cpu().numpy(), inner))):
        nb.grouped_bwd(layer, given, W, on_device(off), dy, dx, dW, torch.zeros(max(nb.grouped_workspace_bytes(layer, n) // 4, 4), device="cuda"))
        want_dx, want_dW = lo.grouped_backward(kept, f64(W), off, f64(dy))
        size_dx, size_dW = lo.grouped_backward(np.abs(kept), sizes[1], off, sizes[2])
        check(dx, want_dx, size_dx, "f32", outer, "dx")
        check(dW, want_dW, size_dW, "f32", n, "dW")


@pytest.mark.parametrize("n,inner,outer,rank", [(8, 64, 64, 8), (200, 64, 64, 8), (600, 100, 104, 20), (17000, 72, 520, 8), (66000, 64, 40, 8)])
def test_adapters_up_to_the_largest_number(n, inner, outer, rank):
    gen = torch.Generator().manual_seed(n + rank)
    small = lambda *shape: torch.randn(*shape, generator=gen).clamp(-3, 3) * 1e-3
    x, dy, W, A, B = small(n, inner), small(n, outer), small(outer, inner), small(3, rank, inner), small(3, outer, rank)
    x[1, inner // 2], dy[0, 2], W[1, 0], A[1, 2, 3], B[2, 4, 1] = LARGEST, -LARGEST, LARGEST, -LARGEST, LARGEST
    x, dy, W, A, B = (t.cuda() for t in (x, dy, W, A, B))
    off, slots, scales = [0, n // 3, n // 2, n], [0, 1, 2], torch.ones(3, device="cuda")
    layer = nb.make_layer("f32", 3, inner, outer, rank=rank, adapters=3)
    y, u, dx = empty(n, outer, outer, "f32"), torch.zeros(n, rank, device="cuda"), empty(n, inner, inner, "f32")
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    nb.adapter_fwd(layer, x, W, A, B, scales, on_device(slots), on_device(off), u, y)
    nb.adapter_bwd(layer, x, W, A, B, scales, on_device(slots), on_device(off), u, dy, dx, dA, dB,
                   torch.zeros(nb.adapter_workspace_bytes(layer, n) // 4, device="cuda"))
    args, sizes = [f64(t) for t in (x, W, A, B)], [np.abs(f64(t)) for t in (x, W, A, B)]
    rest = ([1.0] * 3, slots, off)
    want, size = lo.adapter_forward(*args, *rest), lo.adapter_forward(*sizes, *rest)
    check(u, want[1], size[1], "f32", inner, "u")
    check(y, want[0], size[0], "f32", 2 * inner + rank, "y")
    want, size = lo.adapter_backward(*args, *rest, f64(u), f64(dy)), lo.adapter_backward(*sizes, *rest, np.abs(f64(u)), np.abs(f64(dy)))
    check(dx, want[0], size[0], "f32", 2 * outer + rank, "dx")
    check(dA, want[1], size[1], "f32", n + outer, "dA")
    check(dB, want[2], size[2], "f32", n, "dB")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,inner,outer", [(16, 64, 64), (300, 64, 64), (17000, 72, 520), (8400, 64, 1024), (8400, 1024, 64)])
def test_u_and_v_up_to_the_largest_number_beside_16_bit_matrices(n, inner, outer, dtype):
    """u = v = a scale above bf16's largest number, times 2^-10 in y, dx, dA and dB.  Everything is one product: off by its rounding alone
    (fp16: y and dx are beyond its numbers)."""
    rank, scales = 8, torch.tensor([LARGEST * 0.999], device="cuda")
    want = float(scales.double()) * 2.0 ** -10
    layer = nb.make_layer(dtype, 1, inner, outer, rank=rank, adapters=1)
    new = lambda *shape: torch.zeros(*shape, dtype=TYPES[dtype], device="cuda")
    W, off, workspace = new(outer, inner), on_device([0, n]), torch.zeros(nb.adapter_workspace_bytes(layer, n) // 4, device="cuda")
    near = lambda got, room: bool(torch.all(torch.isinf(got) if got.dtype == torch.float16 else (got.double() / want - 1.0).abs() <= room))
    # u = s in every row; row 5's dy takes it into dB
    x, dy, A, B = new(n, inner), new(n, outer), new(1, rank, inner), new(1, outer, rank)
    x[:, 0], A[0, 0, 0], B[0, :, 0], dy[5, 1] = 1.0, 1.0, 2.0 ** -10, 2.0 ** -10
    u, y = torch.zeros(n, rank, device="cuda"), empty(n, outer, outer, dtype)
    nb.adapter_fwd(layer, x, W, A, B, scales, None, off, u, y)
    assert torch.all(u[:, 0] == scales) and not u[:, 1:].any() and near(y, 2.0 ** -8)
    dA, dB = torch.zeros(A.shape, device="cuda"), torch.zeros(B.shape, device="cuda")
    nb.adapter_bwd(layer, x, W, A, new(1, outer, rank), scales, None, off, u, dy, None, dA, dB, workspace)
    assert near(dB[0, 1, 0], 2.0 ** -23) and dB.count_nonzero() == 1 and not dA.any()
    # v = s in every row; row 5's x takes it into dA
    x, dy, A, B = new(n, inner), new(n, outer), new(1, rank, inner), new(1, outer, rank)
    dy[:, 0], B[0, 0, 0], A[0, 0, :], x[5, 1] = 1.0, 1.0, 2.0 ** -10, 2.0 ** -10
    dx = empty(n, inner, inner, dtype)
    nb.adapter_bwd(layer, x, W, A, B, scales, None, off, torch.zeros_like(u), dy, dx, dA, dB, workspace)
    assert near(dx, 2.0 ** -8) and near(dA[0, 0, 1], 2.0 ** -23) and dA.count_nonzero() == 1 and not dB.any()


# ---- networks --------------------------------------------------------------------------------------------------------------------------

def deep_network(keep8, adapters, seed, **kw):
    rng = np.random.default_rng(seed)
    dims, groups, n = [40, 64, 128, 128, 64, 24, 3], 4, 333
    pairs = list(zip(dims[1:], dims[:-1]))
    draw = lambda *shape: rng.normal(size=shape) * (2.0 / shape[-1]) ** 0.5
    mats = [draw(o, i) if adapters else draw(groups, o, i) for o, i in pairs]
    bank = [(draw(2, 4, i), draw(2, o, 4), np.array([1.0, 0.5])) for o, i in pairs] if adapters else None
    if keep8 is not None:
        kw["keep8"] = keep8
    net = rows_layers.RowNetwork(dims, n, groups, mats, "f32", bank, [0, 1, -1, 0] if adapters else None, **kw)
    x, dy = torch.as_tensor(rng.normal(size=(n, dims[0]))).float().cuda(), torch.as_tensor(rng.normal(size=(n, 3)) * 0.01).float().cuda()
    return net, dims, x, dy, on_device([0, 100, 101, 250, 333])


@pytest.mark.parametrize("adapters", [False, True])
@pytest.mark.parametrize("keep8", [False, True])
def test_deep_networks_whose_layers_share_buffers(keep8, adapters):
    """Six layers: the bits of the same calls with a buffer of its own for everything, for a second batch and its gradients too."""
    net, dims, x, dy, off = deep_network(keep8, adapters, 21)
    n, count = net.n, len(dims) - 1
    for batch in range(2):
        y = net.forward(x, off)
        dx = net.backward(dy, want_dx=True)
        h, inputs, masks, us = x, [], [], []
        for l in range(count):
            blocks = (dims[l] + 31) // 32
            q, e, m = (torch.zeros(n, w, dtype=t, device="cuda") for w, t in ((32 * blocks, torch.int8), (blocks, torch.uint8), (blocks, torch.int32)))
            nb.pack8(h, q, e, m)
            inputs.append((q, e) if keep8 else h)
            masks.append(m if l > 0 else None)
            out, u = torch.zeros(n, dims[l + 1], device="cuda"), torch.zeros(n, 4, device="cuda")
            if adapters:
                nb.adapter_fwd(net.layer[l], h, net.W[l], *net.adapters[l], net.slots, off, u, out)
            else:
                nb.grouped_fwd(net.layer[l], h, net.W[l], off, out)
            us.append(u)
            h = out
        assert torch.equal(y, h)
        d = dy
        for l in reversed(range(count)):
            down, dW, ws = torch.zeros(n, dims[l], device="cuda"), torch.zeros_like(net.dW[l]), torch.zeros_like(net.workspace)
            if adapters:
                A, B, scales = net.adapters[l]
                dA, dB = torch.zeros_like(net.dA[l]), torch.zeros_like(net.dB[l])
                nb.adapter_bwd(net.layer[l], inputs[l], net.W[l], A, B, scales, net.slots, off, us[l], d, down, dA, dB, ws, masks=masks[l])
                nb.grouped_bwd(net.dense[l], inputs[l], None, None, d, None, dW.unsqueeze(0), ws)
                assert torch.equal(dA, net.dA[l]) and torch.equal(dB, net.dB[l]), l
            else:
                nb.grouped_bwd(net.layer[l], inputs[l], net.W[l], off, d, down, dW, ws, masks=masks[l])
            assert torch.equal(dW, net.dW[l]) and dW.any(), l
            d = down
        assert torch.equal(dx, d)
        x, dy = x.flip(0).contiguous(), dy * 2


def test_networks_round_nothing_to_8_bits_unless_told():
    """Gradients of a network made without further arguments are those of its activations as they are (in 8 bits: off by 1e-3 and more)."""
    net, dims, x, dy, off = deep_network(None, False, 22)
    net.forward(x, off)
    net.backward(dy)
    ends, h, kept = off.tolist(), f64(x), []
    for l in range(len(dims) - 1):
        kept.append(h)
        h = lo.grouped_forward(h, f64(net.W[l]), ends, l + 2 < len(dims))
    d = f64(dy)
    for l in reversed(range(len(dims) - 1)):
        d, dW = lo.grouped_backward(kept[l], f64(net.W[l]), ends, d, kept[l] > 0 if l > 0 else None)
        assert np.linalg.norm(f64(net.dW[l]) - dW) <= 5e-6 * np.linalg.norm(dW), l
