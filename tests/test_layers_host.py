"""The layers whose rows choose their matrices, without a GPU: refusals of the library's calls and of the binding, the
oracle's gradients against differences, and what the 8-bit form promises."""
import ctypes as C

import numpy as np
import pytest

from oracle import layers_oracle as lo
from paper_2212_05231_amd import binding as nb

OK = 0x1000


def layer(**kw):
    values = dict(dtype="f32", groups=3, in_dim=20, out_dim=12)
    values.update(kw)
    return nb.make_layer(values.pop("dtype"), values.pop("groups"), values.pop("in_dim"), values.pop("out_dim"), **values)


def grouped_fwd(l, x=OK, W=OK, offsets=OK, n=8, y=OK):
    return nb.lib().neus2_grouped_fwd(C.byref(l), x, W, offsets, n, y, None)


def grouped_bwd(l, x=OK, xq=None, xe=None, masks=None, W=OK, offsets=OK, dy=OK, n=8, dx=OK, dW=OK, ws=OK, size=1 << 30):
    return nb.lib().neus2_grouped_bwd(C.byref(l), x, xq, xe, masks, W, offsets, dy, n, dx, dW, ws, size, None)


def adapter_bwd(l, x=OK, xq=None, xe=None, masks=None, W=OK, A=OK, B=OK, scales=OK, slots=OK, offsets=OK, u=OK, dy=OK, n=8, dx=OK,
                dA=OK, dB=OK, ws=OK, size=1 << 30):
    return nb.lib().neus2_adapter_bwd(C.byref(l), x, xq, xe, masks, W, A, B, scales, slots, offsets, u, dy, n, dx, dA, dB, ws, size, None)


def adapter_fwd(l, **kw):
    v = dict(x=OK, W=OK, A=OK, B=OK, scales=OK, slots=OK, offsets=OK, n=8, u=OK, y=OK)
    v.update(kw)
    return nb.lib().neus2_adapter_fwd(C.byref(l), v["x"], v["W"], v["A"], v["B"], v["scales"], v["slots"], v["offsets"], v["n"], v["u"],
                                      v["y"], None)


def broken(**fields):
    l = layer()
    for name, v in fields.items():
        setattr(l, name, v)
    return l


@pytest.mark.parametrize("fields,code", [
    (dict(dtype=3), -3), (dict(dtype=-1), -3), (dict(groups=0), -3), (dict(groups=(1 << 16) + 1), -3), (dict(in_dim=0), -3),
    (dict(in_dim=65537), -3), (dict(out_dim=0), -3), (dict(out_dim=65537), -3), (dict(x_stride=19), -2), (dict(y_stride=11), -2),
    (dict(x_stride=(1 << 24) + 1), -2), (dict(relu=2), -3), (dict(accumulate=2), -3), (dict(rank=4), -3), (dict(adapters=1), -3)])
def test_descriptors_of_grouped_layers(fields, code):
    l = broken(**fields)
    assert grouped_fwd(l) == code and grouped_bwd(l) == code
    assert len(nb.lib().neus2_last_error()) > 0
    assert nb.grouped_workspace_bytes(l, 100) == -1


@pytest.mark.parametrize("fields,code", [(dict(rank=0), -5), (dict(rank=65), -5), (dict(adapters=0), -3), (dict(adapters=(1 << 16) + 1), -3)])
def test_descriptors_of_adapter_layers(fields, code):
    l = layer(rank=8, adapters=3)
    for name, v in fields.items():
        setattr(l, name, v)
    assert adapter_fwd(l) == code and adapter_bwd(l) == code
    assert nb.adapter_workspace_bytes(l, 100) == -1


def test_pointers_and_sizes_of_grouped_layers():
    l = layer()
    for name in ("x", "W", "offsets", "y"):
        assert grouped_fwd(l, **{name: None}) == -1, name
        assert name.encode() in nb.lib().neus2_last_error()
        assert grouped_fwd(l, **{name: OK + 8}) == -4, name
    assert grouped_fwd(l, n=-1) == -2 and grouped_fwd(l, n=(1 << 28) + 1) == -2
    for name in ("x", "W", "offsets", "dy"):
        assert grouped_bwd(l, **{name: None}) == -1, name
    for name in ("x", "W", "offsets", "dy", "dx", "dW", "masks", "ws"):
        assert grouped_bwd(l, **{name: OK + 4}) == -4, name
    assert grouped_bwd(l, dx=None, dW=None) == -1
    assert grouped_bwd(l, xq=OK, xe=OK) == -3                                     # both forms of the input
    assert grouped_bwd(l, x=None, xq=OK) == -1 and grouped_bwd(l, x=None, xe=OK) == -1
    assert nb.lib().neus2_grouped_fwd(None, OK, OK, OK, 8, OK, None) == -1
    need = nb.grouped_workspace_bytes(l, 1 << 18)
    assert need > 0
    assert grouped_bwd(l, n=1 << 18, size=need - 1) == -2 and grouped_bwd(l, n=1 << 18, ws=None, size=0) == -2
    assert b"workspace" in nb.lib().neus2_last_error()
    wide = layer(dtype="bf16", groups=1 << 16, out_dim=65536, in_dim=65536)          # more workgroups than a launch can have
    assert grouped_bwd(wide, dx=None, n=1 << 16) == -2 and b"workgroups" in nb.lib().neus2_last_error()


def test_pointers_and_sizes_of_adapter_layers():
    l = layer(rank=8, adapters=3)
    for name in ("x", "W", "A", "B", "scales", "offsets", "u", "y"):
        assert adapter_fwd(l, **{name: None}) == -1, name
        assert adapter_fwd(l, **{name: OK + 4}) == -4, name
    assert adapter_fwd(l, slots=OK + 4) == -4 and adapter_fwd(l, n=-1) == -2
    for name in ("x", "W", "A", "B", "scales", "offsets", "u", "dy", "ws"):
        assert adapter_bwd(l, **{name: None}) == -1, name
    for name in ("x", "W", "A", "B", "scales", "slots", "offsets", "u", "dy", "dx", "dA", "dB", "masks", "ws"):
        assert adapter_bwd(l, **{name: OK + 4}) == -4, name
    assert adapter_bwd(l, dA=None) == -1 and adapter_bwd(l, dB=None) == -1
    assert adapter_bwd(l, dx=None, dA=None, dB=None) == -1
    assert adapter_bwd(l, xq=OK, xe=OK) == -3
    need = nb.adapter_workspace_bytes(l, 5000)
    assert adapter_bwd(l, n=5000, size=need - 1) == -2


def test_pack_refusals():
    L = nb.lib()
    pack = lambda dtype=0, x=OK, stride=0, n=8, dim=40, q=OK, e=OK, m=OK: L.neus2_pack8(dtype, x, stride, n, dim, q, e, m, None)
    assert pack(dtype=3) == -3 and pack(dim=0) == -3 and pack(dim=65537) == -3 and pack(stride=39) == -2 and pack(n=-1) == -2
    for name in ("x", "q", "e"):
        assert pack(**{name: None}) == -1, name
        assert pack(**{name: OK + 8}) == -4, name
    assert pack(q=None, e=None, m=None) == -1 and pack(m=OK + 4) == -4
    un = lambda dtype=0, q=OK, e=OK, n=8, dim=40, x=OK, stride=0: L.neus2_unpack8(dtype, q, e, n, dim, x, stride, None)
    assert un(dtype=-1) == -3 and un(stride=39) == -2 and un(n=-1) == -2
    for name in ("q", "e", "x"):
        assert un(**{name: None}) == -1, name
        assert un(**{name: OK + 8}) == -4, name


def test_no_rows_is_no_work():
    """n = 0: nothing to launch forward, and the arrays of rows may be NULL."""
    assert grouped_fwd(layer(), x=None, y=None, n=0) == 0
    assert adapter_fwd(layer(rank=8, adapters=3), x=None, u=None, y=None, n=0) == 0
    assert grouped_bwd(layer(), x=None, dy=None, dx=None, dW=None, ws=None, size=0, n=0) == 0
    assert nb.lib().neus2_pack8(0, None, 0, 0, 40, None, None, None, None) == 0
    assert nb.lib().neus2_unpack8(0, None, None, 0, 40, None, 0, None) == 0


def test_struct_size_against_the_c_compiler(tmp_path):
    import os
    import subprocess
    src, exe = tmp_path / "size.c", tmp_path / "size"
    src.write_text('#include <stdio.h>\n#include "neus2.h"\nint main(void) { printf("%zu\\n", sizeof(neus2_layer)); return 0; }\n')
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run(["gcc", "-I", inc, str(src), "-o", str(exe)], check=True)
    assert int(subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout) == C.sizeof(nb.Neus2Layer)


@pytest.mark.parametrize("groups,inner,outer,rank", [(3, 20, 12, 0), (64, 64, 64, 0), (1, 2048, 4096, 0), (24, 2048, 2048, 64), (49, 64, 64, 8), (1, 512, 512, 0),
                                                     (8, 512, 4096, 0), (300, 512, 512, 0), (2, 257, 300, 0), (7, 40, 64, 0)])
def test_workspace_of_a_batch_serves_every_smaller_one(groups, inner, outer, rank):
    l = layer(groups=groups, in_dim=inner, out_dim=outer, rank=rank, adapters=groups if rank else 0)
    query = nb.adapter_workspace_bytes if rank else nb.grouped_workspace_bytes
    l.dtype = 2 if outer >= 256 else 0
    sizes = [query(l, n) for n in sorted({0, 1, 2, 63, 64, 65, 255, 256, 257, 511, 513, 4095, 4097} | set(range(1000, 300000, 7919)))]
    assert all(a <= b for a, b in zip(sizes, sizes[1:])), sizes


def test_the_binding_names_the_wrong_tensor():
    torch = pytest.importorskip("torch")
    l = layer(groups=2)
    x, W, y = torch.zeros(8, 20), torch.zeros(2, 12, 20), torch.zeros(8, 12)
    off = torch.tensor([0, 3, 8], dtype=torch.int32)
    bad = [("x", dict(x=torch.zeros(8, 21))), ("x", dict(x=x.double())), ("x", dict(x=torch.zeros(20, 8).t())), ("W", dict(W=W[:1])),
           ("W", dict(W=W.half())), ("W", dict(W=torch.zeros(2, 20, 12).transpose(1, 2))), ("offsets", dict(off=off.long())),
           ("offsets", dict(off=off[:2])), ("y", dict(y=torch.zeros(7, 12))), ("y", dict(y=torch.zeros(8, 24)[:, ::2])),
           ("y", dict(y=torch.zeros(8, 16)[:, :12]))]
    for name, change in bad:
        v = dict(x=x, W=W, off=off, y=y)
        v.update(change)
        with pytest.raises(ValueError, match=name):
            nb.grouped_fwd(l, v["x"], v["W"], v["off"], v["y"])
    with pytest.raises(ValueError, match="masks"):
        nb.grouped_bwd(l, x, W, off, y, x, W, masks=torch.zeros(8, 2, dtype=torch.int32))
    with pytest.raises(ValueError, match="xq"):
        nb.grouped_bwd(l, (torch.zeros(8, 20, dtype=torch.int8), torch.zeros(8, 1, dtype=torch.uint8)), W, off, y, x, W)
    with pytest.raises(ValueError, match="rows are"):
        nb.pack8(x.double(), torch.zeros(8, 32, dtype=torch.int8), torch.zeros(8, 1, dtype=torch.uint8))
    with pytest.raises(ValueError, match="e:"):
        nb.pack8(x, torch.zeros(8, 32, dtype=torch.int8), torch.zeros(8, 2, dtype=torch.uint8))
    with pytest.raises(ValueError):
        nb.make_layer("f64", 1, 4, 4)
    with pytest.raises(ValueError, match="host memory"):
        nb.grouped_fwd(l, x, W, off, y)
    with pytest.raises(ValueError, match="workspace"):
        nb.grouped_bwd(l, x, W, off, y, x, W, torch.zeros(64, dtype=torch.float16))
    with pytest.raises(ValueError, match="host memory"):
        nb.pack8(x, torch.zeros(8, 32, dtype=torch.int8), torch.zeros(8, 1, dtype=torch.uint8))


# ---- the oracle itself ---------------------------------------------------------------------------------------------------------

def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(5)
    n, inner, outer, rank = 7, 5, 4, 2
    offsets, slots = [0, 2, 2, 5, 7], [1, 0, -1, 1]
    x, dy = rng.normal(size=(n, inner)), rng.normal(size=(n, outer))
    W = rng.normal(size=(4, outer, inner))
    A, B, c = rng.normal(size=(2, rank, inner)), rng.normal(size=(2, outer, rank)), rng.uniform(0.5, 2, 2)

    def difference(f, t):
        g, h = np.zeros(t.shape), 1e-6
        for i in np.ndindex(t.shape):
            keep = t[i]
            t[i] = keep + h
            up = f()
            t[i] = keep - h
            g[i] = (up - f()) / (2 * h)
            t[i] = keep
        return g
    loss = lambda: float((lo.grouped_forward(x, W, offsets) * dy).sum())
    dx, dW = lo.grouped_backward(x, W, offsets, dy)
    assert np.allclose(dx, difference(loss, x), atol=1e-7) and np.allclose(dW, difference(loss, W), atol=1e-7)
    loss = lambda: float((lo.adapter_forward(x, W[0], A, B, c, slots, offsets)[0] * dy).sum())
    u = lo.adapter_forward(x, W[0], A, B, c, slots, offsets)[1]
    dx, dA, dB = lo.adapter_backward(x, W[0], A, B, c, slots, offsets, u, dy)
    assert np.allclose(dx, difference(loss, x), atol=1e-7)
    assert np.allclose(dA, difference(loss, A), atol=1e-7) and np.allclose(dB, difference(loss, B), atol=1e-7)


def test_the_8_bit_form_is_half_a_step_away_at_most():
    rng = np.random.default_rng(6)
    x = (rng.normal(size=(40, 70)) * np.exp(3 * rng.normal(size=(40, 70)))).astype(np.float32).astype(np.float64)
    q, e, mask = lo.pack8(x, "f32")
    back = lo.unpack8(q, e, 70)
    step = np.repeat(np.ldexp(1.0, e.astype(int) - 127), 32, axis=1)[:, :70]
    assert np.all(np.abs(back - x) <= step / 2) and np.abs(q).max() <= 127 and np.abs(q).reshape(40, 3, 32).max(axis=2).min() >= 63
    assert np.array_equal(mask, x > 0) and not q[:, 70:].any()
    words = lo.mask_words(mask).view(np.uint32)
    assert np.array_equal((words[:, 2] >> 5) & 1, mask[:, 69].astype(np.uint32)) and not (words[:, 2] >> 6).any()


def test_a_refused_backward_call_has_launched_nothing():
    """More workgroups for dW than there are numbers: refused before dx is written, not after (without a GPU that launch would fail first)."""
    l = layer(dtype="bf16", groups=1 << 16, out_dim=65536, in_dim=65536)
    assert grouped_bwd(l, n=1 << 16) == -2 and b"workgroups" in nb.lib().neus2_last_error()


# ---- the network that owns its buffers -----------------------------------------------------------------------------------------

def host_network(dims, n, groups, adapters=False, **kw):
    torch = pytest.importorskip("torch")
    from paper_2212_05231_amd import layers as rows_layers
    pairs = list(zip(dims[1:], dims[:-1]))
    mats = [torch.ones(o, i) if adapters else torch.ones(groups, o, i) for o, i in pairs]
    bank = [(torch.ones(3, 4, i), torch.ones(3, o, 4), torch.ones(3)) for o, i in pairs] if adapters else None
    return rows_layers.RowNetwork(dims, n, groups, mats, "f32", bank, device="cpu", **kw), mats, bank


def held_bytes(thing, seen):
    """Bytes of all tensors that an object, list or tuple holds, every allocation once."""
    torch = pytest.importorskip("torch")
    if isinstance(thing, torch.Tensor):
        storage = thing.untyped_storage()
        new = storage.data_ptr() not in seen
        seen.add(storage.data_ptr())
        return storage.nbytes() if new else 0
    if isinstance(thing, dict):
        thing = list(thing.values())
    return sum(held_bytes(t, seen) for t in thing) if isinstance(thing, (list, tuple)) else 0


@pytest.mark.parametrize("adapters", [False, True])
@pytest.mark.parametrize("dims", [[64] * 9, [40, 64, 128, 128, 64, 24, 3]])
def test_a_network_that_keeps_8_bits_holds_less(dims, adapters):
    """A row costs 9.25 bits a feature kept, beside the input's gradient, the output and two buffers in turn for the activations and for
    their gradients; without 8 bits 32 a feature and a mask."""
    n = 512
    eight, _, _ = host_network(dims, n, 5, adapters, keep8=True)
    full, _, _ = host_network(dims, n, 5, adapters, keep8=False)
    blocks = [(d + 31) // 32 for d in dims]
    masks, ends, turn = 4 * sum(blocks[1:-1]), 4 * (dims[0] + dims[-1]), 4 * max(dims[1:-1])
    rows_of = lambda net: held_bytes([net.rows, net.grad, net.kept or [], net.masks], set())
    assert rows_of(eight) == n * (33 * sum(blocks[:-1]) + masks + ends + 4 * turn)
    assert rows_of(full) == n * (4 * sum(dims[1:-1]) + masks + ends + 2 * turn)
    assert held_bytes(eight.__dict__, set()) < held_bytes(full.__dict__, set())
    # nothing that is still needed lies in the place of something else
    for net in (eight, full):
        for buffers in (net.rows[1:], net.grad[:-1]):
            for a, b in zip(buffers, buffers[1:]):
                assert a.data_ptr() != b.data_ptr() and a.shape[0] == b.shape[0] == n
        assert not {t.data_ptr() for t in net.rows[1:]} & {t.data_ptr() for t in net.grad[:-1]}
        assert all(t.shape[1] == d for t, d in zip(net.rows[1:], dims[1:])) and all(t.shape[1] == d for t, d in zip(net.grad[:-1], dims[:-1]))


def test_a_network_owns_its_matrices():
    """Training steps change the network's matrices, not what it was made from; two networks made from the same tensors share nothing."""
    torch = pytest.importorskip("torch")
    one, mats, bank = host_network([20, 30, 10], 8, 3, True, slots=torch.zeros(3, dtype=torch.int32))
    from paper_2212_05231_amd import layers as rows_layers
    slots = torch.tensor([0, 1, 2], dtype=torch.int32)
    two = rows_layers.RowNetwork([20, 30, 10], 8, 3, [mats[0], mats[1]], "f32", bank, slots, device="cpu")
    given = {t.data_ptr() for t in mats + [t for a in bank for t in a] + [slots]}
    held = [[t.data_ptr() for t in net.W + [t for a in net.adapters for t in a] + [net.slots]] for net in (one, two)]
    assert not given & set(held[0] + held[1]) and not set(held[0]) & set(held[1])
    for t, mat in zip(one.W, mats):
        assert torch.equal(t, mat)
        t.fill_(7.0)
        assert torch.all(mat == 1.0)
