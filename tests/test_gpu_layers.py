"""Layers whose rows choose their matrices on the GPU against their float64 definition (oracle/layers_oracle.py).

Tolerances, from the arithmetic.  A sum of K products p_k is accumulated in fp32: K additions and the instruction's inner sums of
16, each off by at most one unit of 2^-23 of the sum of magnitudes S = sum |p_k|: (K + 32) 2^-23 S.  fp32 factors are three bf16
terms: what is left out of a product is at most 4 * 2^-24 of it, inside the 32.  Two-term factors (u and v of adapters beside 16-bit
matrices) are off by 2^-17, more per product: S 2^-16 for the pair.  The result is rounded to its type: half a step, eps / 2 of its
size, plus half of fp16's smallest number.  For fp32 results the norm of the error is also held to 2e-6 of the result's: products
of two terms instead of three would be off by 2^-17 = 7.6e-6 each.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layers_oracle as lo
from paper_2212_05231_amd import binding as nb
from paper_2212_05231_amd import layers as rows_layers

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
MARK = 7.25                                     # what untouched places hold


def f64(t):
    return t.detach().to("cpu").to(torch.float64).numpy()


def rows(n, width, stride, dtype, gen, scale=1.0, relu=False):
    """[n, width] on the GPU with rows `stride` apart, NaN in between."""
    wide = torch.full((n, stride), float("nan"), dtype=TYPES[dtype])
    t = torch.randn(n, width, generator=gen) * scale
    wide[:, :width] = (t.clamp_min(0) if relu else t).to(TYPES[dtype])
    return wide.cuda()[:, :width]


def empty(n, width, stride, dtype):
    return torch.full((n, stride), MARK, dtype=TYPES[dtype], device="cuda")[:, :width]


def split_rows(n, groups, gen, before=0, behind=0, none=0):
    """offsets of `groups` groups over the rows between the first `before` and the last `behind`."""
    cuts = torch.sort(torch.randint(before, n - behind + 1, (groups - 1,), generator=gen)).values.tolist() if groups > 1 else []
    off = [before] + cuts + [n - behind]
    for g in range(none):                       # some groups without rows
        off[1 + g] = off[g]
    return off


def check(got, want, size, dtype, terms, what, extra=0.0):
    """got against want (NaN where nothing may be written); size: sum of magnitudes of the products, terms: how many."""
    got = f64(got)
    untouched = np.isnan(want)
    assert np.all(got[untouched] == MARK), f"{what}: rows outside the groups written"
    eps = torch.finfo(TYPES[dtype]).eps
    room = (terms + 32) * 2.0 ** -23 * size + extra * size + eps / 2 * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 0.0)
    room = room * 1.001 + 1e-37
    bad = ~(np.abs(got - want) <= room) & ~untouched
    assert not bad.any(), f"{what}: {bad.sum()} off, worst {np.abs(got - want)[bad].max() if bad.any() else 0} at {np.argwhere(bad)[:3]}"
    if dtype == "f32" and extra == 0.0 and np.linalg.norm(want[~untouched]) > 0:
        assert np.linalg.norm((got - want)[~untouched]) <= 2e-6 * np.linalg.norm(want[~untouched]), what


def nan_to(a, value=0.0):
    return np.where(np.isnan(a), value, a)


SHAPES = [  # n, groups, inner, outer, x pad, y pad, before, behind, none
    (1, 1, 1, 1, 0, 0, 0, 0, 0), (1, 1, 64, 64, 0, 0, 0, 0, 0), (5, 3, 33, 7, 0, 0, 1, 1, 1), (48, 3, 200, 130, 0, 0, 0, 0, 1),
    (40, 8, 512, 48, 8, 0, 3, 2, 2), (129, 2, 64, 64, 0, 0, 0, 0, 0), (300, 5, 31, 65, 1, 3, 7, 9, 2), (517, 4, 64, 128, 0, 0, 0, 5, 0),
    (1000, 70, 40, 96, 0, 4, 0, 0, 30), (700, 1, 129, 257, 7, 0, 0, 0, 0), (2051, 3, 256, 320, 0, 0, 2, 0, 1), (900, 2, 1000, 136, 24, 8, 0, 0, 0),
    (4300, 2, 256, 2050, 0, 6, 5, 3, 0), (8300, 64, 512, 512, 0, 0, 0, 0, 5)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:4])))
def test_grouped_forward(shape, dtype):
    n, groups, inner, outer, xp, yp, before, behind, none = shape
    gen = torch.Generator().manual_seed(n + inner)
    off = split_rows(n, groups, gen, before, behind, none)
    x = rows(n, inner, inner + xp, dtype, gen)
    x[:before] = float("nan")                   # rows of nobody: never read into anybody's result
    x[n - behind:] = float("inf")
    W = (torch.randn(groups, outer, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
    for relu in (False, True):
        layer = nb.make_layer(dtype, groups, inner, outer, relu=relu, x_stride=inner + xp, y_stride=outer + yp)
        y = empty(n, outer, outer + yp, dtype)
        nb.grouped_fwd(layer, x, W, offsets, y)
        x64 = f64(x)
        want = lo.grouped_forward(x64, f64(W), off, relu)
        size = lo.grouped_forward(np.abs(nan_to(x64)), np.abs(f64(W)), off)
        check(y, want, size, dtype, inner, "y")
        if yp:
            assert torch.all(y.as_strided((n, yp), (outer + yp, 1), outer) == MARK)         # between the rows


@pytest.mark.parametrize("packed,use_masks,accumulate", [(False, False, 0), (True, True, 1), (True, False, 0), (False, True, 1)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:4])))
def test_grouped_backward(shape, dtype, packed, use_masks, accumulate):
    n, groups, inner, outer, xp, yp, before, behind, none = shape
    gen = torch.Generator().manual_seed(2 * n + inner)
    off = split_rows(n, groups, gen, before, behind, none)
    x = rows(n, inner, inner + xp, dtype, gen, relu=use_masks)
    dy = rows(n, outer, outer + yp, dtype, gen, scale=0.01)
    dy[:before] = float("nan")
    dy[n - behind:] = float("inf")
    W = (torch.randn(groups, outer, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
    q8, e8, mask = lo.pack8(f64(x), dtype)
    x64 = lo.unpack8(q8, e8, inner) if packed else f64(x)
    given = (torch.as_tensor(q8).cuda(), torch.as_tensor(e8).cuda()) if packed else x
    masks = torch.as_tensor(lo.mask_words(mask)).cuda() if use_masks else None
    layer = nb.make_layer(dtype, groups, inner, outer, accumulate=bool(accumulate), x_stride=inner + xp, y_stride=outer + yp)
    ws = nb.grouped_workspace_bytes(layer, n)
    workspace = torch.full((max(ws // 4, 4),), float("nan"), device="cuda")
    want_dx, want_dW = lo.grouped_backward(x64, f64(W), off, f64(dy), mask if use_masks else None)
    size_dx, size_dW = lo.grouped_backward(np.abs(x64), np.abs(f64(W)), off, np.abs(nan_to(f64(dy))))
    dx, dW = empty(n, inner, inner + xp, dtype), torch.full((groups, outer, inner), 0.5, device="cuda")
    nb.grouped_bwd(layer, given, W, offsets, dy, dx, dW, workspace, masks=masks)
    check(dx, want_dx, size_dx, dtype, outer, "dx")
    start = 0.5 if accumulate else 0.0
    most = max(off[g + 1] - off[g] for g in range(groups))
    check(dW, want_dW + start, size_dW + start, "f32", most, "dW", extra=0.0 if not accumulate else 1e-30)
    # one result at a time gives the same bits
    dx2, dW2 = empty(n, inner, inner + xp, dtype), torch.full((groups, outer, inner), 0.5, device="cuda")
    nb.grouped_bwd(layer, None, W, offsets, dy, dx2, None, masks=masks)
    nb.grouped_bwd(layer, given, None, offsets, dy, None, dW2, workspace)
    assert torch.equal(dx2.contiguous(), dx.contiguous()) and torch.equal(dW2, dW)


@pytest.mark.parametrize("packed,use_masks,accumulate", [(False, False, 1), (True, True, 0)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,groups,inner,outer", [(65536, 1, 64, 64), (70011, 20, 64, 64), (66000, 200, 32, 8), (65600, 7, 40, 48)])
def test_narrow_layers_backward_in_one_pass(n, groups, inner, outer, dtype, packed, use_masks, accumulate):
    """Many rows of a narrow layer: runs of rows that begin and end inside groups, groups without rows, rows of nobody; with and
    without dx the same sums."""
    gen = torch.Generator().manual_seed(n)
    off = split_rows(n, groups, gen, 37 if groups > 1 else 0, 41 if groups > 1 else 0, groups // 5)
    x, dy = rows(n, inner, inner, dtype, gen, relu=use_masks), rows(n, outer, outer, dtype, gen, scale=0.01)
    x[:off[0]], dy[:off[0]] = float("nan"), float("inf")
    W = (torch.randn(groups, outer, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    layer = nb.make_layer(dtype, groups, inner, outer, accumulate=bool(accumulate))
    q8, e8, mask = (torch.zeros(n, (inner + 31) // 32 * 32, dtype=torch.int8, device="cuda"),
                    torch.zeros(n, (inner + 31) // 32, dtype=torch.uint8, device="cuda"),
                    torch.zeros(n, (inner + 31) // 32, dtype=torch.int32, device="cuda"))
    nb.pack8(x, q8, e8, mask)                                    # held to the definition by test_pack_and_unpack
    x64 = lo.unpack8(q8.cpu().numpy(), e8.cpu().numpy(), inner) if packed else f64(x)
    workspace = torch.full((nb.grouped_workspace_bytes(layer, n) // 4,), float("nan"), device="cuda")
    dx, dW = empty(n, inner, inner, dtype), torch.full((groups, outer, inner), 0.5, device="cuda")
    given, masks = (q8, e8) if packed else x, mask if use_masks else None
    nb.grouped_bwd(layer, given, W, on_device(off), dy, dx, dW, workspace, masks=masks)
    want_dx, want_dW = lo.grouped_backward(x64, f64(W), off, f64(dy), f64(x) > 0 if use_masks else None)
    size_dx, size_dW = lo.grouped_backward(np.abs(nan_to(x64)), np.abs(f64(W)), off, np.abs(np.where(np.isinf(f64(dy)), 0.0, f64(dy))))
    check(dx, want_dx, size_dx, dtype, outer, "dx")
    start = 0.5 if accumulate else 0.0
    most = max(off[g + 1] - off[g] for g in range(groups))
    check(dW, want_dW + start, size_dW + start, "f32", most, "dW", extra=0.0 if not accumulate else 1e-30)
    dW2, dx2 = torch.full((groups, outer, inner), 0.5, device="cuda"), empty(n, inner, inner, dtype)
    nb.grouped_bwd(layer, given, None, on_device(off), dy, None, dW2, workspace)
    nb.grouped_bwd(layer, None, W, on_device(off), dy, dx2, None, masks=masks)
    assert torch.equal(dW, dW2) and torch.equal(dx, dx2)


def test_one_group_without_offsets_and_many_chunks():
    """offsets NULL; 70 000 rows of a small matrix: hundreds of chunks joined in order, bit for bit the same twice."""
    gen = torch.Generator().manual_seed(3)
    n, inner, outer = 70001, 38, 64
    x, dy = rows(n, inner, inner, "f32", gen), rows(n, outer, outer, "f32", gen, 0.01)
    W = torch.randn(1, outer, inner, generator=gen).cuda()
    layer = nb.make_layer("f32", 1, inner, outer)
    workspace = torch.zeros(nb.grouped_workspace_bytes(layer, n) // 4, device="cuda")
    results = []
    for _ in range(2):
        dx, dW, y = empty(n, inner, inner, "f32"), torch.zeros(1, outer, inner, device="cuda"), empty(n, outer, outer, "f32")
        nb.grouped_fwd(layer, x, W, None, y)
        nb.grouped_bwd(layer, x, W, None, dy, dx, dW, workspace)
        results.append((y, dx, dW))
    want_dx, want_dW = lo.grouped_backward(f64(x), f64(W), None, f64(dy))
    size_dx, size_dW = lo.grouped_backward(np.abs(f64(x)), np.abs(f64(W)), None, np.abs(f64(dy)))
    check(results[0][1], want_dx, size_dx, "f32", outer, "dx")
    check(results[0][2], want_dW, size_dW, "f32", n, "dW")
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_infinities_and_nan_stay_in_their_rows():
    gen = torch.Generator().manual_seed(4)
    for dtype in ("f32", "f16", "bf16"):
        x = rows(200, 72, 72, dtype, gen)
        W = (torch.randn(2, 40, 72, generator=gen) * 0.1).to(TYPES[dtype]).cuda()
        offsets = torch.tensor([0, 90, 200], dtype=torch.int32, device="cuda")
        layer = nb.make_layer(dtype, 2, 72, 40, relu=True)
        y, z = empty(200, 40, 40, dtype), empty(200, 40, 40, dtype)
        nb.grouped_fwd(layer, x, W, offsets, y)
        x[17, 3], x[100, 71] = float("nan"), float("inf")
        nb.grouped_fwd(layer, x, W, offsets, z)
        assert torch.isnan(z[17]).all() and (torch.isnan(z[100]) | torch.isinf(z[100]) | (z[100] == 0)).all()
        keep = [r for r in range(200) if r not in (17, 100)]
        assert torch.equal(y[keep], z[keep])


@pytest.mark.parametrize("n,inner,outer,rank", [(40, 64, 48, 8), (300, 64, 64, 8), (600, 256, 256, 16), (600, 64, 320, 40)])
def test_an_infinite_adapter_stays_with_its_rows(n, inner, outer, rank):
    """Segments that share tiles: what is not finite in one adapter's matrices reaches its own rows and gradients only."""
    for dtype in ("f32", "f16", "bf16"):
        gen = torch.Generator().manual_seed(n + rank)
        x, dy = rows(n, inner, inner, dtype, gen), rows(n, outer, outer, dtype, gen, 0.01)
        W = (torch.randn(outer, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
        A = (torch.randn(3, rank, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
        B = (torch.randn(3, outer, rank, generator=gen) * rank ** -0.5).to(TYPES[dtype]).cuda()
        scales = torch.ones(3, device="cuda")
        off, slots = [0, n // 3 + 1, n // 2 + 1, n], [0, 1, 2]
        layer = nb.make_layer(dtype, 3, inner, outer, rank=rank, adapters=3)
        workspace = torch.zeros(nb.adapter_workspace_bytes(layer, n) // 4, device="cuda")
        results = []
        for poison in (False, True):
            if poison:
                A[1, 0, 0], B[1, 1, 0], B[1, 2, 1] = float("nan"), float("inf"), -float("inf")
            y, u, dx = empty(n, outer, outer, dtype), torch.zeros(n, rank, device="cuda"), empty(n, inner, inner, dtype)
            dA, dB = torch.zeros(A.shape, device="cuda"), torch.zeros(B.shape, device="cuda")
            nb.adapter_fwd(layer, x, W, A, B, scales, on_device(slots), on_device(off), u, y)
            nb.adapter_bwd(layer, x, W, A, B, scales, on_device(slots), on_device(off), u, dy, dx, dA, dB, workspace)
            results.append((y, u, dx, dA, dB))
        others = torch.ones(n, dtype=torch.bool)
        others[off[1]:off[2]] = False
        for a, b in zip(results[0][:3], results[1][:3]):
            assert torch.equal(a[others.cuda()], b[others.cuda()]) and not torch.equal(a, b)
        for a, b in zip(results[0][3:], results[1][3:]):
            assert torch.equal(a[[0, 2]], b[[0, 2]]) and not torch.equal(a[1], b[1])


def test_more_groups_than_rows():
    """5000 groups for 300 rows, most of them without any."""
    gen = torch.Generator().manual_seed(6)
    n, inner, outer, groups = 300, 40, 24, 5000
    off = torch.sort(torch.randint(0, n + 1, (groups - 1,), generator=gen)).values.tolist()
    off = [0] + off + [n]
    x, dy = rows(n, inner, inner, "bf16", gen), rows(n, outer, outer, "bf16", gen, 0.01)
    W = (torch.randn(groups, outer, inner, generator=gen) * inner ** -0.5).bfloat16().cuda()
    layer = nb.make_layer("bf16", groups, inner, outer)
    y, dx, dW = empty(n, outer, outer, "bf16"), empty(n, inner, inner, "bf16"), torch.ones(groups, outer, inner, device="cuda")
    need = nb.grouped_workspace_bytes(layer, n) // 4
    nb.grouped_fwd(layer, x, W, on_device(off), y)
    nb.grouped_bwd(layer, x, W, on_device(off), dy, dx, dW, torch.zeros(need, device="cuda") if need else None)
    magnitudes = [np.abs(f64(t)) for t in (x, W, dy)]
    want_dx, want_dW = lo.grouped_backward(f64(x), f64(W), off, f64(dy))
    size_dx, size_dW = lo.grouped_backward(magnitudes[0], magnitudes[1], off, magnitudes[2])
    check(y, lo.grouped_forward(f64(x), f64(W), off), lo.grouped_forward(magnitudes[0], magnitudes[1], off), "bf16", inner, "y")
    check(dx, want_dx, size_dx, "bf16", outer, "dx")
    check(dW, want_dW, size_dW, "f32", n, "dW")


def test_wrong_offsets_stay_inside_the_arrays():
    """Offsets beyond the rows, negative or decreasing: results are whatever they are, but only inside the outputs."""
    gen = torch.Generator().manual_seed(5)
    n, inner, outer, groups = 300, 40, 72, 4
    x, dy = rows(n, inner, inner, "bf16", gen), rows(n, outer, outer, "bf16", gen)
    W = torch.randn(groups, outer, inner, generator=gen).bfloat16().cuda()
    layer = nb.make_layer("bf16", groups, inner, outer)
    for off in ([0, 10 ** 9, 10 ** 9, 2 ** 31 - 1, 5], [-5, 100, 50, 300, 0], [300, 0, 300, 0, 300], [2 ** 31 - 1, -2 ** 31, 0, 300, 299]):
        offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
        guard = torch.full((n + 64, outer), MARK, dtype=torch.bfloat16, device="cuda")
        back = torch.full((n + 64, inner), MARK, dtype=torch.bfloat16, device="cuda")
        need = nb.grouped_workspace_bytes(layer, n) // 4
        workspace = torch.full((need + 256,), MARK, device="cuda")
        dW = torch.full((groups + 1, outer, inner), MARK, device="cuda")
        nb.grouped_fwd(layer, x, W, offsets, guard[32:n + 32])
        nb.grouped_bwd(layer, x, W, offsets, dy, back[32:n + 32], dW[:groups], workspace[:need] if need else None)
        torch.cuda.synchronize()
        for t in (guard, back):
            assert torch.all(t[:32] == MARK) and torch.all(t[n + 32:] == MARK)
        assert torch.all(dW[groups] == MARK) and torch.all(workspace[need:] == MARK)


@pytest.mark.parametrize("n,groups,inner,outer,dtype", [(65600, 64, 64, 64, "f16"), (65600, 64, 64, 48, "f32"), (9000, 64, 512, 512, "bf16"),
                                                        (700, 300, 256, 320, "bf16")])
def test_wrong_offsets_stay_inside_the_arrays_of_every_kernel(n, groups, inner, outer, dtype):
    """Groups that each claim all rows, or none: more tiles, units and chunks than there is room for."""
    gen = torch.Generator().manual_seed(groups)
    x, dy = rows(n, inner, inner, dtype, gen), rows(n, outer, outer, dtype, gen)
    W = torch.randn(groups, outer, inner, generator=gen).to(TYPES[dtype]).cuda()
    layer = nb.make_layer(dtype, groups, inner, outer)
    rank, slots = 8, 5
    adapted = nb.make_layer(dtype, groups, inner, outer, rank=rank, adapters=slots)
    A, B = torch.randn(slots, rank, inner, generator=gen).to(TYPES[dtype]).cuda(), torch.randn(slots, outer, rank, generator=gen).to(TYPES[dtype]).cuda()
    scales, named = torch.ones(slots, device="cuda"), on_device([g % 7 - 1 for g in range(groups)])
    q, e = torch.zeros(n, (inner + 31) // 32 * 32, dtype=torch.int8, device="cuda"), torch.full((n, (inner + 31) // 32), 127, dtype=torch.uint8, device="cuda")
    for off in ([0 if g % 2 else n for g in range(groups + 1)], [n if g % 2 else 0 for g in range(groups + 1)], [2 ** 31 - 1] * (groups + 1)):
        offsets = on_device(off)
        y, dx = (torch.full((n + 64, w), MARK, dtype=TYPES[dtype], device="cuda") for w in (outer, inner))
        u = torch.full((n + 64, rank), MARK, device="cuda")
        dW, dA, dB = (torch.full((k + 1, *shape), MARK, device="cuda") for k, shape in ((groups, (outer, inner)), (slots, (rank, inner)), (slots, (outer, rank))))
        sizes = [nb.grouped_workspace_bytes(layer, n) // 4, nb.adapter_workspace_bytes(adapted, n) // 4]
        spaces = [torch.full((s + 256,), MARK, device="cuda") for s in sizes]
        nb.grouped_fwd(layer, x, W, offsets, y[32:n + 32])
        for given in (x, (q, e)):
            nb.grouped_bwd(layer, given, W, offsets, dy, dx[32:n + 32], dW[:groups], spaces[0][:sizes[0]] if sizes[0] else None)
        nb.adapter_fwd(adapted, x, W[0], A, B, scales, named, offsets, u[32:n + 32], y[32:n + 32])
        nb.adapter_bwd(adapted, x, W[0], A, B, scales, named, offsets, u[32:n + 32], dy, dx[32:n + 32], dA[:slots], dB[:slots], spaces[1][:sizes[1]])
        torch.cuda.synchronize()
        for t in (y, dx, u):
            assert torch.all(t[:32] == MARK) and torch.all(t[n + 32:] == MARK)
        for t in (dW, dA, dB):
            assert torch.all(t[-1] == MARK)
        for t, s in zip(spaces, sizes):
            assert torch.all(t[s:] == MARK)


ADAPTERS = [  # n, groups, slots, inner, outer, rank, pad, before, behind
    (1, 1, 1, 1, 1, 1, 0, 0, 0), (3, 3, 2, 40, 20, 4, 0, 0, 0), (64, 64, 9, 200, 72, 16, 0, 0, 0), (61, 5, 3, 96, 136, 5, 3, 4, 3),
    (65, 65, 40, 64, 64, 8, 0, 0, 0), (500, 7, 7, 64, 64, 8, 0, 3, 9), (700, 3, 5, 136, 200, 64, 8, 0, 0), (1500, 100, 30, 300, 129, 33, 1, 1, 1),
    (2000, 2, 2, 640, 64, 16, 0, 0, 0), (900, 9, 4, 256, 300, 20, 0, 5, 0), (1100, 150, 6, 320, 512, 64, 0, 0, 2)]


def adapter_case(shape, dtype, seed):
    n, groups, slots, inner, outer, rank, pad, before, behind = shape
    gen = torch.Generator().manual_seed(seed)
    off = split_rows(n, groups, gen, before, behind) if n != groups else list(range(n + 1))
    named = torch.randint(-1, slots, (groups,), generator=gen)
    if groups > 2:
        named[0], named[1] = slots + 3, 0                       # beyond the bank: none; the first adapter twice or more
        named[2] = 0
    if groups == 1:
        named[0] = 0
    x = rows(n, inner, inner + pad, dtype, gen, relu=True)
    W = (torch.randn(outer, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    A = (torch.randn(slots, rank, inner, generator=gen) * inner ** -0.5).to(TYPES[dtype]).cuda()
    B = (torch.randn(slots, outer, rank, generator=gen) * rank ** -0.5).to(TYPES[dtype]).cuda()
    scales = (torch.rand(slots, generator=gen) + 0.5).cuda()
    return off, named.tolist(), x, W, A, B, scales, gen


def on_device(ints):
    return torch.tensor(ints, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", ADAPTERS, ids=lambda s: "x".join(map(str, s[:6])))
def test_adapter_forward(shape, dtype):
    n, groups, slots, inner, outer, rank, pad, before, behind = shape
    off, named, x, W, A, B, scales, gen = adapter_case(shape, dtype, n + rank)
    layer = nb.make_layer(dtype, groups, inner, outer, rank=rank, adapters=slots, relu=rank % 2 == 0, x_stride=inner + pad, y_stride=outer + pad)
    for listed in (named, None):
        y, u = empty(n, outer, outer + pad, dtype), torch.full((n, rank), MARK, device="cuda")
        nb.adapter_fwd(layer, x, W, A, B, scales, None if listed is None else on_device(listed), on_device(off), u, y)
        want_y, want_u = lo.adapter_forward(f64(x), f64(W), f64(A), f64(B), f64(scales), listed, off, rank % 2 == 0)
        ax = [np.abs(f64(t)) for t in (x, W, A, B)]
        size_y, size_u = lo.adapter_forward(nan_to(ax[0]), *ax[1:], f64(scales), listed, off)
        check(u, want_u, size_u, "f32", inner, "u")
        check(y, want_y, size_y, dtype, 2 * inner + rank, "y", extra=0.0 if dtype == "f32" else 2.0 ** -16)


@pytest.mark.parametrize("packed,use_masks,accumulate", [(False, False, 1), (True, True, 0), (True, False, 1)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", ADAPTERS, ids=lambda s: "x".join(map(str, s[:6])))
def test_adapter_backward(shape, dtype, packed, use_masks, accumulate):
    n, groups, slots, inner, outer, rank, pad, before, behind = shape
    off, named, x, W, A, B, scales, gen = adapter_case(shape, dtype, n + 2 * rank)
    dy = rows(n, outer, outer + pad, dtype, gen, 0.01)
    dy[:before] = float("nan")
    if not use_masks:
        x *= torch.randn(x.shape, generator=gen).sign().to(TYPES[dtype]).cuda()
    q8, e8, mask = lo.pack8(f64(x), dtype)
    x64 = lo.unpack8(q8, e8, inner) if packed else f64(x)
    u = torch.as_tensor(nan_to(lo.adapter_forward(x64, f64(W), f64(A), f64(B), f64(scales), named, off)[1])).float().cuda()
    layer = nb.make_layer(dtype, groups, inner, outer, rank=rank, adapters=slots, accumulate=bool(accumulate), x_stride=inner + pad,
                          y_stride=outer + pad)
    workspace = torch.full((max(nb.adapter_workspace_bytes(layer, n) // 4, 4),), float("nan"), device="cuda")
    given = (torch.as_tensor(q8).cuda(), torch.as_tensor(e8).cuda()) if packed else x
    masks = torch.as_tensor(lo.mask_words(mask)).cuda() if use_masks else None
    dx = empty(n, inner, inner + pad, dtype)
    dA, dB = torch.full(A.shape, 0.5, device="cuda"), torch.full(B.shape, 0.5, device="cuda")
    nb.adapter_bwd(layer, given, W, A, B, scales, on_device(named), on_device(off), u, dy, dx, dA, dB, workspace, masks=masks)
    args = (f64(W), f64(A), f64(B), f64(scales), named, off)
    want = lo.adapter_backward(x64, *args, f64(u), f64(dy), mask if use_masks else None)
    size = lo.adapter_backward(np.abs(x64), *(np.abs(a) for a in args[:3]), *args[3:], np.abs(f64(u)), np.abs(nan_to(f64(dy))))
    two = 0.0 if dtype == "f32" else 2.0 ** -16
    start = 0.5 if accumulate else 0.0
    check(dx, want[0], size[0], dtype, 2 * outer + rank, "dx", extra=two)
    check(dA, want[1] + start, size[1] + start, "f32", n + outer, "dA", extra=two or (1e-30 if accumulate else 0.0))
    check(dB, want[2] + start, size[2] + start, "f32", n, "dB", extra=two or (1e-30 if accumulate else 0.0))
    dx2 = empty(n, inner, inner + pad, dtype)
    nb.adapter_bwd(layer, None, W, A, B, scales, on_device(named), on_device(off), None, dy, dx2, None, None, workspace, masks=masks)
    dA2, dB2 = torch.full(A.shape, 0.5, device="cuda"), torch.full(B.shape, 0.5, device="cuda")
    nb.adapter_bwd(layer, given, None, A, B, scales, on_device(named), on_device(off), u, dy, None, dA2, dB2, workspace)
    assert torch.equal(dx.contiguous(), dx2.contiguous()) and torch.equal(dA, dA2) and torch.equal(dB, dB2)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,dim,pad", [(1, 1, 0), (3, 31, 0), (70, 32, 0), (33, 33, 5), (50, 200, 0), (200, 64, 8), (5, 1001, 3)])
def test_pack_and_unpack(n, dim, pad, dtype):
    """Every step and every exponent equal to the definition's: nothing is rounded but the steps themselves."""
    gen = torch.Generator().manual_seed(n + dim)
    x = rows(n, dim, dim + pad, dtype, gen)
    x *= torch.exp2(torch.randint(-12, 6, (n, dim), generator=gen).float()).to(TYPES[dtype]).cuda()
    top = torch.finfo(TYPES[dtype]).max
    special = [0.0, -0.0, top, -top, top * 0.99, torch.finfo(TYPES[dtype]).tiny, torch.finfo(TYPES[dtype]).smallest_normal / 4, 127.0, 127.5,
               -127.5, 0.5, 1.5, 2.5, float("inf"), float("nan"), -float("inf"), 255.0 / 256]
    for i, v in enumerate(special):
        if i < n:
            x[i, (7 * i) % dim] = v
    if n > 20:
        x[19], x[20] = 0.0, torch.finfo(TYPES[dtype]).tiny
    blocks = (dim + 31) // 32
    q = torch.full((n, 32 * blocks), 77, dtype=torch.int8, device="cuda")
    e = torch.full((n, blocks), 77, dtype=torch.uint8, device="cuda")
    m = torch.full((n, blocks), 77, dtype=torch.int32, device="cuda")
    nb.pack8(x, q, e, m)
    want_q, want_e, mask = lo.pack8(f64(x), dtype)
    assert np.array_equal(e.cpu().numpy(), want_e)
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(m.cpu().numpy(), lo.mask_words(mask))
    back = empty(n, dim, dim + pad, dtype)
    nb.unpack8(q, e, back)
    assert np.array_equal(f64(back), lo.unpack8(want_q, want_e, dim), equal_nan=True)
    alone = torch.zeros_like(m)
    nb.pack8(x, None, None, alone)
    assert torch.equal(alone, m)
    if pad:
        assert torch.all(back.as_strided((n, pad), (dim + pad, 1), dim) == MARK)


def test_no_rows():
    dev = dict(device="cuda")
    layer = nb.make_layer("f32", 2, 8, 4)
    x, y, W = torch.zeros(0, 8, **dev), torch.zeros(0, 4, **dev), torch.ones(2, 4, 8, **dev)
    off, dW = torch.zeros(3, dtype=torch.int32, **dev), torch.ones(2, 4, 8, **dev)
    nb.grouped_fwd(layer, x, W, off, y)
    nb.grouped_bwd(layer, x, W, off, y, x, dW)
    assert not dW.any()
    a = nb.make_layer("f32", 2, 8, 4, rank=2, adapters=3)
    A, B, s = torch.ones(3, 2, 8, **dev), torch.ones(3, 4, 2, **dev), torch.ones(3, **dev)
    dA, dB, u = torch.ones(3, 2, 8, **dev), torch.ones(3, 4, 2, **dev), torch.zeros(0, 2, **dev)
    ws = torch.zeros(nb.adapter_workspace_bytes(a, 0) // 4, **dev)
    nb.adapter_fwd(a, x, W[0], A, B, s, None, off, u, y)
    nb.adapter_bwd(a, x, W[0], A, B, s, None, off, u, y, x, dA, dB, ws)
    assert not dA.any() and not dB.any()
    # groups without rows among rows of nobody
    x, y = torch.ones(300, 8, **dev), torch.full((300, 4), MARK, **dev)
    off = on_device([40, 40, 40])
    dW = torch.ones(2, 4, 8, **dev)
    nb.grouped_fwd(layer, x, W, off, y)
    nb.grouped_bwd(layer, x, W, off, y, None, dW, torch.zeros(max(nb.grouped_workspace_bytes(layer, 300) // 4, 4), **dev))
    assert torch.all(y == MARK) and not dW.any()


def test_offsets_beyond_31_bits():
    """1.1 million rows of 2048 fp16 values: the last rows begin behind 2^31 values, 2^32 bytes."""
    n, inner, outer = 1_100_003, 2048, 16
    x = torch.zeros(n, inner, dtype=torch.float16, device="cuda")
    gen = torch.Generator().manual_seed(8)
    tail = torch.randn(50, inner, generator=gen).half()
    x[-50:] = tail.cuda()
    W = (torch.randn(2, outer, inner, generator=gen) * inner ** -0.5).half().cuda()
    dy = torch.zeros(n, outer, dtype=torch.float16, device="cuda")
    dy[-50:] = torch.randn(50, outer, generator=gen).half().cuda()
    off = [0, n - 30, n]
    layer = nb.make_layer("f16", 2, inner, outer)
    y = empty(n, outer, outer, "f16")
    nb.grouped_fwd(layer, x, W, on_device(off), y)
    cut = [0, 20, 50]
    want = lo.grouped_forward(f64(x[-50:]), f64(W), cut)
    check(y[-50:], want, lo.grouped_forward(np.abs(f64(x[-50:])), np.abs(f64(W)), cut), "f16", inner, "y")
    assert not y[:-50].any()
    dW = torch.zeros(2, outer, inner, device="cuda")
    workspace = torch.zeros(max(nb.grouped_workspace_bytes(layer, n) // 4, 4), device="cuda")
    dx = torch.zeros_like(x)
    nb.grouped_bwd(layer, x, W, on_device(off), dy, dx, dW, workspace)
    magnitudes = [np.abs(f64(t)) for t in (tail, W, dy[-50:])]
    want_dx, want_dW = lo.grouped_backward(f64(tail), f64(W), cut, f64(dy[-50:]))
    size_dx, size_dW = lo.grouped_backward(magnitudes[0], magnitudes[1], cut, magnitudes[2])
    check(dx[-50:], want_dx, size_dx, "f16", outer, "dx")
    check(dW, want_dW, size_dW, "f32", 50, "dW")                               # all other rows are zero: exact


def make_network(dtype, adapters, keep8, seed):
    rng = np.random.default_rng(seed)
    dims, groups, n = [38, 64, 64, 3], 5, 333                    # the colour network's widths
    off = [0, 100, 100, 101, 250, 333]
    scale = lambda o, i: rng.normal(size=(o, i)) * (2.0 / i) ** 0.5
    if adapters:
        mats = [scale(dims[l + 1], dims[l]) for l in range(3)]
        bank = [(np.stack([scale(4, dims[l]) for _ in range(3)]), np.stack([scale(dims[l + 1], 4) for _ in range(3)]), np.array([1.0, 0.5, 2.0]))
                for l in range(3)]
        slots = [0, 1, -1, 2, 0]
    else:
        mats = [np.stack([scale(dims[l + 1], dims[l]) for _ in range(groups)]) for l in range(3)]
        bank, slots = None, None
    return rows_layers.RowNetwork(dims, n, groups, mats, dtype, bank, slots, keep8=keep8), rng, off


def reference_step(net, x, off, dy):
    """The network's outputs and gradients in float64.  Where it keeps 8-bit inputs the gradients are those of the values it has kept
    (fp32 and fp64 activations can fall on two sides of a tie: one step of 2^-6 in a norm of 100 is 1.5e-4), each of which has to lie
    within half a step of the float64 one."""
    kept, masks, us, h = [], [], [], f64(x)
    W = [f64(w) for w in net.W]
    adapters = [[f64(t) for t in a] for a in net.adapters] if net.adapters else None
    slots = None if net.slots is None else net.slots.cpu().tolist()
    for l in range(3):
        masks.append(h > 0)
        kept.append(h)
        if net.keep8:
            q, e = (t.cpu().numpy() for t in net.kept[l])
            step = np.repeat(np.ldexp(1.0, e.astype(np.int64) - 127), 32, axis=1)[:, :h.shape[1]]
            kept[l] = lo.unpack8(q, e, h.shape[1])
            assert np.all(np.abs(kept[l] - h) <= step * (0.5 + 1e-3))
        if adapters:
            h, u = lo.adapter_forward(h, W[l], *adapters[l], slots, off, l < 2)
            us.append(u)
        else:
            h = lo.grouped_forward(h, W[l], off, l < 2)
    y, grads, d = h, {"dW": [None] * 3, "dA": [None] * 3, "dB": [None] * 3}, f64(dy)
    for l in reversed(range(3)):
        mask = masks[l] if l > 0 else None
        if adapters:
            grads["dW"][l] = d.T @ kept[l]
            d, grads["dA"][l], grads["dB"][l] = lo.adapter_backward(kept[l], W[l], *adapters[l], slots, off, us[l], d, mask)
        else:
            d, grads["dW"][l] = lo.grouped_backward(kept[l], W[l], off, d, mask)
    return y, d, grads


@pytest.mark.parametrize("adapters", [False, True])
@pytest.mark.parametrize("keep8", [False, True])
def test_a_network_of_them_forward_backward_and_adam(adapters, keep8):
    """Three layers with the colour network's widths, chained as a program does: outputs, every gradient and one Adam step."""
    net, rng, off = make_network("f32", adapters, keep8, 11)
    x = torch.as_tensor(rng.normal(size=(net.n, 38))).float().cuda()
    dy = torch.as_tensor(rng.normal(size=(net.n, 3)) * 0.01).float().cuda()
    y = net.forward(x, on_device(off))
    dx = net.backward(dy, want_dx=True)
    want_y, want_dx, grads = reference_step(net, x, off, dy)
    rel = lambda a, b: np.linalg.norm(f64(a) - b) / np.linalg.norm(b)
    assert rel(y, want_y) <= 1e-6 and rel(dx, want_dx) <= 5e-6
    for l in range(3):
        assert rel(net.dW[l], grads["dW"][l]) <= 5e-6, l
        if adapters:
            assert rel(net.dA[l], grads["dA"][l]) <= 5e-6 and rel(net.dB[l], grads["dB"][l]) <= 5e-6, l
    net.init_optimizer(lr=1e-2)
    before, g = f64(net.W[1]), f64(net.dW[1])
    net.adam()
    assert np.allclose(before - f64(net.W[1]), np.where(g == 0, 0.0, 1e-2 * np.sign(g)), atol=1e-6)   # the first step of Adam: lr * sign


def test_gradients_of_a_network_against_differences():
    """d loss / d theta of the whole chain against central differences of the float64 network, inputs kept as they are."""
    net, rng, off = make_network("f32", True, False, 12)
    x = torch.as_tensor(rng.normal(size=(net.n, 38))).float().cuda()
    dy = torch.as_tensor(rng.normal(size=(net.n, 3))).float().cuda()
    net.forward(x, on_device(off))
    net.backward(dy)
    def loss():
        return float((reference_step(net, x, off, dy)[0] * f64(dy)).sum())
    for t, grad in ((net.W[0], net.dW[0]), (net.adapters[1][0], net.dA[1]), (net.adapters[0][1], net.dB[0])):
        i = tuple(np.unravel_index(int(grad.abs().argmax()), grad.shape))
        keep, h = float(t[i]), 2.0 ** -10
        t[i] = keep + h
        up = loss()
        t[i] = keep - h
        down = loss()
        t[i] = keep
        got = float(grad[i])
        # the loss is piecewise linear or quadratic in one weight except where a mask flips
        assert abs((up - down) / (2 * h) - got) <= 2e-2 * abs(got) + 1e-3


def test_captured_steps_replay():
    """A training step of a network in a HIP graph, beside eager steps of another one that shares nothing, and two graphs that
    share one workspace, replayed in turn: every replay the eager step's bits."""
    net, rng, off = make_network("f32", True, True, 13)
    other, _, _ = make_network("f32", True, True, 13)
    x = torch.as_tensor(rng.normal(size=(net.n, 38))).float().cuda()
    dy = torch.as_tensor(rng.normal(size=(net.n, 3)) * 0.01).float().cuda()
    offsets = on_device(off)
    want_y = other.forward(x, offsets).clone()
    other.backward(dy)
    want = [t.clone() for t in other.dW + other.dA + other.dB]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        net.forward(x, offsets)
        net.backward(dy)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    forward, backward = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(forward):
        y = net.forward(x, offsets)
    with torch.cuda.graph(backward):
        net.backward(dy)
    for replay in range(4):
        for t in net.dW + net.dA + net.dB + [y]:
            t.fill_(MARK)
        net.workspace.fill_(-1)
        other.forward(x * 2, offsets)
        other.backward(dy)
        torch.cuda.synchronize()
        forward.replay()
        backward.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want_y), replay
        for got, w in zip(net.dW + net.dA + net.dB, want):
            assert torch.equal(got, w), replay


def test_on_another_stream():
    """Calls go to the current stream: work queued before them on it is waited for, other streams are not needed."""
    gen = torch.Generator().manual_seed(9)
    n, inner, outer = 4000, 512, 256
    x = rows(n, inner, inner, "bf16", gen)
    W = (torch.randn(1, outer, inner, generator=gen) * inner ** -0.5).bfloat16().cuda()
    layer = nb.make_layer("bf16", 1, inner, outer)
    want = empty(n, outer, outer, "bf16")
    nb.grouped_fwd(layer, x, W, None, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    late, y = torch.zeros_like(x), empty(n, outer, outer, "bf16")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            late.copy_(x * 0.5)
        late.copy_(x)
        nb.grouped_fwd(layer, late, W, None, y)
    side.synchronize()
    assert torch.equal(y, want)
