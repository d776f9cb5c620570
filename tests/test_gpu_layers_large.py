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


# ---- the kernels of large calls ------------------------------------------------------------------------------------------------------------
# On 256 compute units: workgroups that take a second tile (narrow ones from 98304 rows on, wide ones from 257 tiles of 256 x 256 on) and
# the quarters of a last round; tiles of 128 x 64 and 128 x 128 (512 of them); outputs of more and of less than 32 MB.

GROUPED = [  # dtypes, n, groups, inner, outer, pad, before, behind, none
    ("f32", 140003, 20, 64, 64, 0, 0, 0, 3), ("f32 f16", 110000, 300, 40, 24, 8, 77, 130, 60), ("f16 bf16", 270000, 20, 64, 64, 0, 0, 0, 0),
    ("f32 bf16", 66000, 3, 100, 48, 0, 0, 5, 0), ("f32 f16", 66000, 3, 48, 100, 4, 0, 0, 0),
    ("f32", 17000, 4, 72, 520, 0, 9, 0, 0), ("f32", 17000, 4, 520, 72, 0, 0, 0, 1), ("f16", 33000, 2, 72, 520, 8, 0, 0, 0),
    ("f16 bf16", 20000, 1, 64, 1024, 0, 0, 0, 0), ("bf16", 20000, 1, 1024, 64, 0, 0, 0, 0), ("f16 bf16", 20000, 5, 192, 1000, 0, 100, 33, 1),
    ("f16 bf16", 20000, 5, 1000, 192, 8, 100, 33, 1), ("bf16", 20000, 6, 128, 1032, 8, 0, 0, 0), ("f16", 20000, 6, 1032, 128, 0, 0, 0, 0),
    ("f16 bf16", 34000, 3, 64, 264, 0, 0, 300, 0), ("f16", 34000, 3, 264, 64, 0, 0, 0, 0)]


@pytest.mark.parametrize("dtype,shape", [(t, s[1:]) for s in GROUPED for t in s[0].split()], ids=lambda v: v if isinstance(v, str) else "x".join(map(str, v[:4])))
def test_grouped_rows_of_large_calls(shape, dtype):
    n, groups, inner, outer, pad, before, behind, none = shape
    gen = torch.Generator().manual_seed(n + inner)
    off = split_rows(n, groups, gen, before, behind, none) if groups > 1 else [0, n]
    x, dy = rows(n, inner, inner + pad, dtype, gen), rows(n, outer, outer + pad, dtype, gen, 0.01)
    for t in (x, dy):
        t[:before], t[n - behind:] = float("nan"), float("inf")
    W = (torch.randn(groups, outer, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    layer = nb.make_layer(dtype, groups, inner, outer, relu=True, x_stride=inner + pad, y_stride=outer + pad)
    kept = torch.rand(n, inner, generator=gen) < 0.5
    masks = torch.as_tensor(lo.mask_words(kept.numpy())).cuda()
    y, dx = empty(n, outer, outer + pad, dtype), empty(n, inner, inner + pad, dtype)
    nb.grouped_fwd(layer, x, W, on_device(off), y)
    nb.grouped_bwd(layer, None, W, on_device(off), dy, dx, None, masks=masks)
    for t, width in ((y, outer), (dx, inner)):
        assert pad == 0 or torch.all(t.as_strided((n, pad), (width + pad, 1), width) == MARK)
    only = lambda a: np.where(np.isfinite(a), a, 0.0)                  # rows of nobody
    check(y, lo.grouped_forward(f64(x), f64(W), off, True), lo.grouped_forward(np.abs(only(f64(x))), np.abs(f64(W)), off), dtype, inner, "y")
    # dx of rows is the forward product of dy with the transposed matrices
    Wt = f64(W).transpose(0, 2, 1)
    want, size = lo.grouped_forward(f64(dy), Wt, off), lo.grouped_forward(np.abs(only(f64(dy))), np.abs(Wt), off)
    check(dx, np.where(kept.numpy() | np.isnan(want), want, 0.0), size, dtype, outer, "dx")


@pytest.mark.parametrize("dtype,n,groups,inner,outer,accumulate", [("f32", 140003, 20, 64, 64, 0), ("f16", 270000, 20, 64, 64, 1), ("bf16", 270000, 7, 56, 40, 0)])
def test_narrow_gradients_of_large_calls(dtype, n, groups, inner, outer, accumulate):
    """Both gradients in one pass, dx of more than 32 MB (the last case less), inputs in 8 bits and masks."""
    gen = torch.Generator().manual_seed(n)
    off = split_rows(n, groups, gen, 50, 70, 2)
    x, dy = rows(n, inner, inner, dtype, gen, relu=True), rows(n, outer, outer, dtype, gen, 0.01)
    W = (torch.randn(groups, outer, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    blocks = (inner + 31) // 32
    q, e, masks = (torch.zeros(n, w, dtype=t, device="cuda") for w, t in ((32 * blocks, torch.int8), (blocks, torch.uint8), (blocks, torch.int32)))
    nb.pack8(x, q, e, masks)
    x64 = lo.unpack8(q.cpu().numpy(), e.cpu().numpy(), inner)
    layer = nb.make_layer(dtype, groups, inner, outer, accumulate=bool(accumulate))
    workspace = torch.full((nb.grouped_workspace_bytes(layer, n) // 4,), float("nan"), device="cuda")
    dx, dW = empty(n, inner, inner, dtype), torch.randn(groups, outer, inner, generator=gen).cuda()
    start = f64(dW) if accumulate else 0.0
    nb.grouped_bwd(layer, (q, e), W, on_device(off), dy, dx, dW, workspace, masks=masks)
    want_dx, want_dW = lo.grouped_backward(x64, f64(W), off, f64(dy), f64(x) > 0)
    size_dx, size_dW = lo.grouped_backward(np.abs(x64), np.abs(f64(W)), off, np.abs(f64(dy)))
    check(dx, want_dx, size_dx, dtype, outer, "dx")
    check(dW, want_dW + start, size_dW + np.abs(start), "f32", max(b - a for a, b in zip(off, off[1:])), "dW")


@pytest.mark.parametrize("packed,accumulate", [(False, 1), (True, 0)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,groups,inner,outer", [(8300, 64, 264, 304), (66000, 1, 304, 264), (70000, 3, 296, 520)])
def test_wide_sums_of_partly_filled_tiles(n, groups, inner, outer, dtype, packed, accumulate):
    """dW in tiles of 256 x 256 that end inside the matrix, less than 32 MB of them; groups of one chunk and of many."""
    gen = torch.Generator().manual_seed(n)
    off = split_rows(n, groups, gen, 3, 5, 1) if groups > 1 else [0, n]
    x, dy = rows(n, inner, inner + 8, dtype, gen), rows(n, outer, outer, dtype, gen, 0.01)
    layer = nb.make_layer(dtype, groups, inner, outer, accumulate=bool(accumulate), x_stride=inner + 8)
    blocks = (inner + 31) // 32
    q, e = torch.zeros(n, 32 * blocks, dtype=torch.int8, device="cuda"), torch.zeros(n, blocks, dtype=torch.uint8, device="cuda")
    nb.pack8(x, q, e)
    x64 = lo.unpack8(q.cpu().numpy(), e.cpu().numpy(), inner) if packed else f64(x)
    dW = torch.randn(groups, outer, inner, generator=gen).cuda()
    start = f64(dW) if accumulate else 0.0
    workspace = torch.full((max(nb.grouped_workspace_bytes(layer, n) // 4, 4),), float("nan"), device="cuda")
    nb.grouped_bwd(layer, (q, e) if packed else x, None, on_device(off), dy, None, dW, workspace)
    want, size, dy64 = np.zeros(dW.shape), np.zeros(dW.shape), f64(dy)
    for g in range(groups):
        part = slice(off[g], off[g + 1])
        want[g], size[g] = dy64[part].T @ x64[part], np.abs(dy64[part]).T @ np.abs(x64[part])
    check(dW, want + start, size + np.abs(start), "f32", max(b - a for a, b in zip(off, off[1:])), "dW")


ADAPTED = [  # dtypes, n, groups, slots, inner, outer, rank, pad, before, behind
    ("f32 f16 bf16", 66000, 49, 30, 64, 64, 8, 0, 0, 9), ("f32 f16", 17000, 9000, 5, 72, 520, 20, 0, 4, 0), ("f32 bf16", 17000, 40, 12, 520, 72, 16, 0, 0, 0),
    ("f16 bf16", 8400, 150, 40, 64, 1024, 16, 8, 0, 0), ("f16 bf16", 8400, 4200, 7, 1024, 64, 20, 0, 10, 20), ("bf16", 16500, 3, 3, 128, 1024, 33, 0, 0, 0),
    ("f16", 16500, 24, 20, 1024, 128, 64, 0, 5, 5), ("f16 bf16", 8400, 24, 6, 192, 1000, 64, 0, 0, 100), ("bf16", 8400, 24, 6, 1000, 192, 12, 0, 0, 0)]


def large_adapters(shape, dtype, seed):
    n, groups, slots, inner, outer, rank, pad, before, behind = shape
    gen = torch.Generator().manual_seed(seed)
    off, named = split_rows(n, groups, gen, before, behind), torch.randint(-1, slots + 1, (groups,), generator=gen)
    x, dy = rows(n, inner, inner + pad, dtype, gen), rows(n, outer, outer + pad, dtype, gen, 0.01)
    W = (torch.randn(outer, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    A = (torch.randn(slots, rank, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    B = (torch.randn(slots, outer, rank, generator=gen) * rank ** -0.5).to(TYPES[dtype]).cuda()
    return off, named.tolist(), x, dy, W, A, B, (torch.rand(slots, generator=gen) + 0.5).cuda(), gen


@pytest.mark.parametrize("dtype,shape", [(t, s[1:]) for s in ADAPTED for t in s[0].split()], ids=lambda v: v if isinstance(v, str) else "x".join(map(str, v[:6])))
def test_adapters_of_large_calls(shape, dtype):
    """Tiles of 128 x 64, 128 x 128 and 256 x 256 that hold parts of segments, whole ones and more than 64 of them; forward and every gradient."""
    n, groups, slots, inner, outer, rank, pad, before, behind = shape
    off, named, x, dy, W, A, B, scales, gen = large_adapters(shape, dtype, n + rank)
    layer = nb.make_layer(dtype, groups, inner, outer, rank=rank, adapters=slots, relu=True, x_stride=inner + pad, y_stride=outer + pad)
    y, u, dx = empty(n, outer, outer + pad, dtype), torch.full((n, rank), MARK, device="cuda"), empty(n, inner, inner + pad, dtype)
    kept = torch.rand(n, inner, generator=gen) < 0.5
    masks = torch.as_tensor(lo.mask_words(kept.numpy())).cuda()
    nb.adapter_fwd(layer, x, W, A, B, scales, on_device(named), on_device(off), u, y)
    args, sizes = [f64(t) for t in (W, A, B, scales)], [np.abs(f64(t)) for t in (W, A, B, scales)]
    want, size = lo.adapter_forward(f64(x), *args, named, off, True), lo.adapter_forward(np.abs(f64(x)), *sizes, named, off)
    check(u, want[1], size[1], "f32", inner, "u")
    check(y, want[0], size[0], dtype, 2 * inner + rank, "y")
    dA, dB = torch.zeros(A.shape, device="cuda"), torch.zeros(B.shape, device="cuda")
    workspace = torch.full((nb.adapter_workspace_bytes(layer, n) // 4,), float("nan"), device="cuda")
    nb.adapter_bwd(layer, x, W, A, B, scales, on_device(named), on_device(off), u, dy, dx, dA, dB, workspace, masks=masks)
    want, size = lo.adapter_backward(f64(x), *args, named, off, f64(u), f64(dy), kept.numpy()), lo.adapter_backward(
        np.abs(f64(x)), *sizes, named, off, np.abs(f64(u)), np.abs(f64(dy)))
    check(dx, want[0], size[0], dtype, 2 * outer + rank, "dx")
    check(dA, want[1], size[1], "f32", n + outer, "dA")
    check(dB, want[2], size[2], "f32", n, "dB")


@pytest.mark.parametrize("dtype,n,inner,outer,rank", [("f32", 66000, 64, 64, 8), ("f32", 17000, 72, 520, 20), ("f32", 17000, 520, 72, 20), ("f16", 17000, 72, 520, 20),
                                                      ("f16", 8400, 64, 1024, 16), ("bf16", 8400, 1024, 64, 16), ("bf16", 8400, 64, 1024, 40)])
def test_an_infinite_adapter_stays_with_its_rows_in_large_tiles(dtype, n, inner, outer, rank):
    gen = torch.Generator().manual_seed(n + rank)
    x, dy = rows(n, inner, inner, dtype, gen), rows(n, outer, outer, dtype, gen, 0.01)
    W = (torch.randn(outer, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    A = (torch.randn(3, rank, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    B = (torch.randn(3, outer, rank, generator=gen) * rank ** -0.5).to(TYPES[dtype]).cuda()
    scales, off, slots = torch.ones(3, device="cuda"), [0, n // 3 + 1, n // 3 + 90, n // 3 + 100, n], [0, 1, 2, 0]
    layer = nb.make_layer(dtype, 4, inner, outer, rank=rank, adapters=3)
    workspace, results = torch.zeros(nb.adapter_workspace_bytes(layer, n) // 4, device="cuda"), []
    for poison in (False, True):
        if poison:
            A[1, 0, 0], B[1, 1, 0], B[1, 2, 1] = float("nan"), float("inf"), -float("inf")
        y, u, dx = empty(n, outer, outer, dtype), torch.zeros(n, rank, device="cuda"), empty(n, inner, inner, dtype)
        dA, dB = torch.zeros(A.shape, device="cuda"), torch.zeros(B.shape, device="cuda")
        nb.adapter_fwd(layer, x, W, A, B, scales, on_device(slots), on_device(off), u, y)
        nb.adapter_bwd(layer, x, W, A, B, scales, on_device(slots), on_device(off), u, dy, dx, dA, dB, workspace)
        results.append((y, u, dx, dA, dB))
    others = torch.ones(n, dtype=torch.bool, device="cuda")
    others[off[1]:off[2]] = False
    for a, b in zip(results[0][:3], results[1][:3]):
        assert torch.equal(a[others], b[others]) and not torch.isfinite(b[~others]).all(1).any()
    for a, b in zip(results[0][3:], results[1][3:]):
        assert torch.equal(a[[0, 2]], b[[0, 2]]) and not torch.isfinite(b[1]).all()


@pytest.mark.parametrize("dtype,n,groups,inner,outer,rank", [("f32", 110000, 64, 64, 40, 8), ("f16", 20000, 64, 64, 1024, 16), ("bf16", 20000, 64, 1024, 64, 16),
                                                             ("f32", 17000, 300, 72, 520, 20), ("f32", 17000, 300, 520, 72, 20)])
def test_wrong_offsets_stay_inside_the_arrays_of_large_calls(dtype, n, groups, inner, outer, rank):
    """Groups that each claim all rows, none, or rows that do not exist, in the kernels of the tests above."""
    gen = torch.Generator().manual_seed(groups)
    x, dy = rows(n, inner, inner, dtype, gen), rows(n, outer, outer, dtype, gen)
    W = torch.randn(groups, outer, inner, generator=gen).to(TYPES[dtype]).cuda()
    A, B = torch.randn(5, rank, inner, generator=gen).to(TYPES[dtype]).cuda(), torch.randn(5, outer, rank, generator=gen).to(TYPES[dtype]).cuda()
    layer, adapted = nb.make_layer(dtype, groups, inner, outer), nb.make_layer(dtype, groups, inner, outer, rank=rank, adapters=5)
    scales, named = torch.ones(5, device="cuda"), on_device([g % 7 - 1 for g in range(groups)])
    sizes = [nb.grouped_workspace_bytes(layer, n) // 4, nb.adapter_workspace_bytes(adapted, n) // 4]
    wild = torch.randint(-2 ** 31, 2 ** 31 - 1, (groups + 1,), generator=gen).tolist()
    for off in ([0 if g % 2 else n for g in range(groups + 1)], [n if g % 2 else 0 for g in range(groups + 1)], [0] + wild[1:-1] + [n], wild):
        offsets = on_device(off)
        y, dx = (torch.full((n + 64, w), MARK, dtype=TYPES[dtype], device="cuda") for w in (outer, inner))
        u = torch.full((n + 64, rank), MARK, device="cuda")
        dW, dA, dB = (torch.full((k + 1, *shape), MARK, device="cuda") for k, shape in ((groups, (outer, inner)), (5, (rank, inner)), (5, (outer, rank))))
        spaces = [torch.full((s + 256,), MARK, device="cuda") for s in sizes]
        nb.grouped_fwd(layer, x, W, offsets, y[32:n + 32])
        nb.grouped_bwd(layer, x, W, offsets, dy, dx[32:n + 32], dW[:groups], spaces[0][:sizes[0]] if sizes[0] else None)
        nb.adapter_fwd(adapted, x, W[0], A, B, scales, named, offsets, u[32:n + 32], y[32:n + 32])
        nb.adapter_bwd(adapted, x, W[0], A, B, scales, named, offsets, u[32:n + 32], dy, dx[32:n + 32], dA[:5], dB[:5], spaces[1][:sizes[1]])
        torch.cuda.synchronize()
        for t in (y, dx, u):
            assert torch.all(t[:32] == MARK) and torch.all(t[n + 32:] == MARK)
        for t in (dW, dA, dB):
            assert torch.all(t[-1] == MARK)
        for t, s in zip(spaces, sizes):
            assert torch.all(t[s:] == MARK)
