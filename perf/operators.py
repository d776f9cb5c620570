"""Layers of bias-free networks whose rows choose their matrices, as a user's program calls them: products grouped by frame,
view or block of space, low-rank adapters beside a shared matrix, and layer inputs kept in 8 bits for the backward pass.

A case is a dict of plain values.  `prepare` makes what a program holds before the call (samples or tokens in their groups,
matrices, what the forward pass kept, output buffers), `run` makes one pass.  With `own` false a pass is computed in plain
torch operations in 32 bits; with `own` true by the library's calls.  Widths are those of the framework's networks (16 to 64)
or generic ones; row counts are those of its batches (rays times samples) down to single rows.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _case(name, kind, **values):
    return dict(values, name=name, kind=kind)


def listed():
    return [
        # rows grouped by expert: two rows for each of eight matrices, one step of an interactive program
        _case("grouped-fwd-tokens", "grouped_fwd", dtype="bf16", n=16, groups=8, inner=1024, outer=1024),
        # one hidden layer of a network per frame: 20 frames of a dynamic scene, 4096 rays x 64 samples
        _case("grouped-fwd-frames", "grouped_fwd", dtype="f32", n=262144, groups=20, inner=64, outer=64, relu=True),
        # odd widths, rows cut out of wider ones, groups without rows
        _case("grouped-fwd-odd", "grouped_fwd", dtype="f16", n=5003, groups=13, inner=200, outer=333, pad=8, empty=4),
        # wide layers, where the matrix cores bound the pass
        _case("grouped-fwd-wide", "grouped_fwd", dtype="bf16", n=16384, groups=8, inner=2048, outer=4096),
        # the hidden layer of the 20 frames backwards, its input kept in 8 bits and its ReLU's masks in bits
        _case("grouped-bwd-frames", "grouped_bwd", dtype="f32", n=262144, groups=20, inner=64, outer=64, packed=True, masks=True),
        # the wide layer backwards: both gradients
        _case("grouped-bwd-wide", "grouped_bwd", dtype="bf16", n=16384, groups=8, inner=2048, outer=4096),
        # the hidden activations of the largest batch (16384 rays x 64 samples) put away and taken back
        _case("pack-samples", "pack", dtype="f32", n=1048576, inner=64),
        # wide activations of an odd width
        _case("pack-wide", "pack", dtype="bf16", n=4099, inner=2000),
        # one row for each of 64 requests, adapters drawn from a bank, some the same, some requests without one
        _case("adapter-fwd-tokens", "adapter_fwd", dtype="bf16", n=64, groups=64, slots=40, inner=2048, outer=2048, rank=16),
        # the rows of 24 requests at once
        _case("adapter-fwd-prompts", "adapter_fwd", dtype="f16", n=8192, groups=24, slots=16, inner=2048, outer=2048, rank=64),
        # a shared hidden layer with an adapter for each of 49 views, trained on 2048 rays x 64 samples
        _case("adapter-bwd-views", "adapter_bwd", dtype="f32", n=131072, groups=49, slots=49, inner=64, outer=64, rank=8, masks=True),
        # adapters of a wide layer trained for 16 requests, its input kept in 8 bits
        _case("adapter-bwd-wide", "adapter_bwd", dtype="bf16", n=8192, groups=16, slots=16, inner=2048, outer=2048, rank=16, packed=True),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["grouped_fwd", "grouped_fwd", "grouped_bwd", "grouped_bwd", "pack", "adapter_fwd", "adapter_fwd", "adapter_bwd"])
    case = {"kind": kind, "dtype": rng.choice(["f32", "f16", "bf16"]), "n": _log_int(rng, 1, 262144), "inner": _log_int(rng, 16, 2048)}
    if rng.random() < 0.5:
        case["inner"] = max(16, case["inner"] // 16 * 16)
    if kind == "pack":
        case["n"] = max(1, min(case["n"] * 4, (1 << 26) // case["inner"]))
        return case
    case["outer"] = _log_int(rng, 16, 4096)
    if rng.random() < 0.5:
        case["outer"] = max(16, case["outer"] // 16 * 16)
    most = 1 << (34 if case["dtype"] == "f32" else 36)
    case["n"] = max(1, min(case["n"], most // (case["inner"] * case["outer"])))
    case["groups"] = min(_log_int(rng, 1, 64), max(1, (1 << 27) // (case["inner"] * case["outer"])))
    if rng.random() < 0.3:
        case["pad"] = rng.randint(1, 24)
    if rng.random() < 0.3:
        case["empty"] = rng.randint(0, case["groups"] // 2)
    if kind.startswith("adapter"):
        case["rank"] = rng.choice([4, 8, 16, 16, 32, 64])
        case["slots"] = rng.randint(1, case["groups"] + 4)
    if kind.endswith("fwd"):
        case["relu"] = rng.random() < 0.5
    else:
        case["packed"] = rng.random() < 0.5
        case["masks"] = rng.random() < 0.5
    return case


# ---- inputs -----------------------------------------------------------------------------------------------------------------

def _split_rows(case, gen):
    """Row counts of the groups: uneven ones, some of them none."""
    n, groups = case["n"], case["groups"]
    if n == groups:
        return list(range(groups + 1))
    share = torch.rand(groups, generator=gen, dtype=torch.float64) + 0.5
    if case.get("empty"):
        share[torch.randperm(groups, generator=gen)[:min(case["empty"], groups - 1)]] = 0.0
    ends = torch.round(torch.cumsum(share, 0) / share.sum() * n).to(torch.int64)
    ends[-1] = n
    return [0] + ends.tolist()


def _rows(n, width, pad, dtype, gen, relu=False):
    """[n, width] of a type; with `pad` the columns of a wider array.  `relu`: the output of one, half of it zeros."""
    t = torch.randn(n, width + pad, generator=gen, device="cuda")
    if relu:
        t = t.clamp_min(0.0)
    return t.to(dtype)[:, :width]


def _blocks(x):
    """fp32 copy of x [n, width] as [n, ceil(width / 32), 32], zeros behind the last column."""
    n, width = x.shape
    full = torch.zeros(n, (width + 31) // 32 * 32, device=x.device)
    full[:, :width] = x.float()
    return full.view(n, -1, 32)


def _pack_plain(x):
    """The 8-bit form of x: q int8 [n, 32 * blocks], e uint8 [n, blocks], masks int32 [n, blocks] (bit c: x > 0).  A block's
    exponent t is the smallest (at least -126) at which the largest magnitude rounds to at most 127 steps of 2^t; e = t + 127,
    or 255 where the block holds a value that is not finite."""
    b = _blocks(x)
    n, blocks = b.shape[:2]
    top = b.abs().amax(2)
    finite = torch.isfinite(b).all(2)
    mantissa, power = torch.frexp(torch.where(finite, top, torch.zeros_like(top)))
    t = (power - 7 + (mantissa >= 127.5 / 128).int()).clamp_min(-126)
    t = torch.where(mantissa == 0, torch.full_like(t, -126), t)
    inverse = ((127 - t) << 23).view(torch.float32)
    # at the type's last power of two the 64th step is beyond its largest number
    most = torch.where(t == (10 if x.dtype == torch.float16 else 122), 63.0, 127.0)[..., None]
    q = torch.minimum(torch.maximum(torch.round(b * inverse[..., None]), -most), most)
    q = torch.where(finite[..., None], q, torch.zeros_like(q)).to(torch.int8)
    e = torch.where(finite, t + 127, torch.full_like(t, 255)).to(torch.uint8)
    bits = (b > 0).to(torch.int64) << torch.arange(32, device=x.device)
    masks = bits.sum(2)
    masks = torch.where(masks >= 1 << 31, masks - (1 << 32), masks).to(torch.int32)
    return q.reshape(n, -1), e, masks


def _unpack_plain(q, e, width, dtype):
    scale = torch.where(e == 255, float("nan"), (e.int() << 23).view(torch.float32))
    return (q.view(q.shape[0], -1, 32).float() * scale[..., None]).view(q.shape[0], -1)[:, :width].to(dtype)


def _bools(masks, width):
    bits = (masks[..., None] >> torch.arange(32, device=masks.device, dtype=torch.int32)) & 1
    return bits.view(masks.shape[0], -1)[:, :width] != 0


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _prepare_own(s)
    return s


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dtype, n, inner = TYPES[case["dtype"]], case["n"], case["inner"]
    kind, pad = case["kind"], case.get("pad", 0)
    s = {"case": case, "dtype": dtype}
    if kind == "pack":
        # activations of samples: a feature's spread differs from block to block
        x = _rows(n, inner, 0, torch.float32, gen, relu=True) * torch.exp(2.0 * torch.randn(1, inner, generator=gen, device="cuda"))
        s["x"] = x.to(dtype).contiguous()
    else:
        outer, groups = case["outer"], case["groups"]
        s["ends"] = _split_rows(case, host)
        s["offsets"] = torch.tensor(s["ends"], dtype=torch.int32, device="cuda")
        s["x"] = _rows(n, inner, pad, dtype, gen, relu=True)
        count = groups if kind.startswith("grouped") else 1
        s["W"] = (torch.randn(count, outer, inner, generator=gen, device="cuda") * (2.0 / inner) ** 0.5).to(dtype)
        if kind.startswith("adapter"):
            rank, slots = case["rank"], case["slots"]
            s["W"] = s["W"][0]
            s["A"] = (torch.randn(slots, rank, inner, generator=gen, device="cuda") * inner ** -0.5).to(dtype)
            s["B"] = (torch.randn(slots, outer, rank, generator=gen, device="cuda") * (0.1 / rank) ** 0.5).to(dtype)
            s["scales"] = torch.rand(slots, generator=gen, device="cuda") + 0.5
            if slots == groups:
                s["slot_list"] = torch.randperm(slots, generator=host).tolist()
            else:
                s["slot_list"] = torch.randint(-1, slots, (groups,), generator=host).tolist()
            s["slots"] = torch.tensor(s["slot_list"], dtype=torch.int32, device="cuda")
        if kind.endswith("bwd"):
            s["dy"] = _rows(n, outer, pad, dtype, gen) * 0.01
            if pad:
                wide = torch.zeros(n, outer + pad, dtype=dtype, device="cuda")
                wide[:, :outer] = s["dy"]
                s["dy"] = wide[:, :outer]
            if case.get("packed") or case.get("masks"):
                q, e, masks = _pack_plain(s["x"])
                if case.get("packed"):
                    s["packed"] = (q, e)
                if case.get("masks"):
                    s["masks"] = masks
            if kind == "adapter_bwd":
                s["u"] = torch.zeros(n, case["rank"], device="cuda")
                x = _kept(s).float()
                for g, slot in enumerate(s["slot_list"]):
                    lo, hi = s["ends"][g], s["ends"][g + 1]
                    if slot >= 0 and hi > lo:
                            s["u"][lo:hi] = (x[lo:hi] @ s["A"][slot].float().t()) * s["scales"][slot]
    return s


def _kept(s):
    """The layer's input as the backward pass has it."""
    if "packed" in s:
        return _unpack_plain(*s["packed"], s["case"]["inner"], s["dtype"])
    return s["x"]


def _prepare_own(s):
    """The buffers and the descriptor that a program keeps from step to step."""
    from paper_2212_05231_amd import binding as nb
    case, dtype, x = s["case"], s["dtype"], s["x"]
    n, inner = x.shape
    f32 = dict(dtype=torch.float32, device="cuda")
    kind = case["kind"]
    if kind == "pack":
        blocks = (inner + 31) // 32
        s["q"] = torch.zeros(n, 32 * blocks, dtype=torch.int8, device="cuda")
        s["e"] = torch.zeros(n, blocks, dtype=torch.uint8, device="cuda")
        s["bits"] = torch.zeros(n, blocks, dtype=torch.int32, device="cuda")
        s["back"] = torch.zeros(n, inner, dtype=dtype, device="cuda")
        return
    outer, pad = case["outer"], case.get("pad", 0)
    s["layer"] = nb.make_layer(case["dtype"], case["groups"], inner, outer, rank=case.get("rank", 0), adapters=case.get("slots", 0),
                               relu=case.get("relu", False), x_stride=inner + pad, y_stride=outer + pad)
    wide = lambda width: torch.zeros(n, width + pad, dtype=dtype, device="cuda")[:, :width]
    if kind.endswith("fwd"):
        s["y"] = wide(outer)
        s["u"] = torch.zeros(n, case["rank"], **f32) if kind == "adapter_fwd" else None
        return
    s["dx"] = wide(inner)
    if kind == "grouped_bwd":
        s["dW"] = torch.zeros(case["groups"], outer, inner, **f32)
        size = nb.grouped_workspace_bytes(s["layer"], n)
    else:
        s["dA"], s["dB"] = torch.zeros(s["A"].shape, **f32), torch.zeros(s["B"].shape, **f32)
        size = nb.adapter_workspace_bytes(s["layer"], n)
    s["workspace"] = torch.zeros(max(size // 4, 4), dtype=torch.int32, device="cuda")


# ---- one pass ---------------------------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2212_05231_amd import binding as nb
    kind, n = s["case"]["kind"], s["x"].shape[0]
    if kind == "pack":
        nb.pack8(s["x"], s["q"], s["e"], s["bits"])
        nb.unpack8(s["q"], s["e"], s["back"])
        return {"back": s["back"], "masks": _bools(s["bits"], s["x"].shape[1])}
    layer = s["layer"]
    if kind == "grouped_fwd":
        nb.grouped_fwd(layer, s["x"], s["W"], s["offsets"], s["y"])
        return {"y": s["y"]}
    if kind == "adapter_fwd":
        nb.adapter_fwd(layer, s["x"], s["W"], s["A"], s["B"], s["scales"], s["slots"], s["offsets"], s["u"], s["y"])
        return {"y": s["y"], "u": s["u"]}
    x = s.get("packed", s["x"])
    if kind == "grouped_bwd":
        nb.grouped_bwd(layer, x, s["W"], s["offsets"], s["dy"], s["dx"], s["dW"], s["workspace"], masks=s.get("masks"))
        return {"dx": s["dx"], "dW": s["dW"]}
    nb.adapter_bwd(layer, x, s["W"], s["A"], s["B"], s["scales"], s["slots"], s["offsets"], s["u"], s["dy"], s["dx"], s["dA"], s["dB"],
                   s["workspace"], masks=s.get("masks"))
    return {"dx": s["dx"], "dA": s["dA"], "dB": s["dB"]}


def _run_plain(s):
    case, dtype, x = s["case"], s["dtype"], s["x"]
    kind = case["kind"]
    if kind == "pack":
        q, e, masks = _pack_plain(x)
        return {"back": _unpack_plain(q, e, x.shape[1], dtype), "masks": _bools(masks, x.shape[1])}
    n, ends, groups = x.shape[0], s["ends"], case["groups"]
    spans = [(g, ends[g], ends[g + 1]) for g in range(groups) if ends[g + 1] > ends[g]]
    f32 = dict(dtype=torch.float32, device="cuda")
    if kind == "grouped_fwd":
        y = torch.empty(n, case["outer"], **f32)
        for g, lo, hi in spans:
            y[lo:hi] = x[lo:hi].float() @ s["W"][g].float().t()
        return {"y": (y.clamp_min(0.0) if case.get("relu") else y).to(dtype)}
    if kind == "adapter_fwd":
        xf = x.float()
        y, u = xf @ s["W"].float().t(), torch.zeros(n, case["rank"], **f32)
        for g, lo, hi in spans:
            slot = s["slot_list"][g]
            if slot >= 0:
                u[lo:hi] = (xf[lo:hi] @ s["A"][slot].float().t()) * s["scales"][slot]
                y[lo:hi] += u[lo:hi] @ s["B"][slot].float().t()
        return {"y": (y.clamp_min(0.0) if case.get("relu") else y).to(dtype), "u": u}
    kept, dy = _kept(s).float(), s["dy"].float()
    if kind == "grouped_bwd":
        dx, dW = torch.empty(n, case["inner"], **f32), torch.zeros(s["W"].shape, **f32)
        for g, lo, hi in spans:
            dx[lo:hi] = dy[lo:hi] @ s["W"][g].float()
            dW[g] = dy[lo:hi].t() @ kept[lo:hi]
        grads = {"dW": dW}
    else:
        dx = dy @ s["W"].float()
        dA, dB = torch.zeros(s["A"].shape, **f32), torch.zeros(s["B"].shape, **f32)
        for g, lo, hi in spans:
            slot = s["slot_list"][g]
            if slot >= 0:
                v = (dy[lo:hi] @ s["B"][slot].float()) * s["scales"][slot]
                dx[lo:hi] += v @ s["A"][slot].float()
                dA[slot] += v.t() @ kept[lo:hi]
                dB[slot] += dy[lo:hi].t() @ s["u"][lo:hi]
        grads = {"dA": dA, "dB": dB}
    if case.get("masks"):
        dx = torch.where(_bools(s["masks"], case["inner"]), dx, torch.zeros_like(dx))
    return dict({"dx": dx.to(dtype)}, **grads)


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------------

def exact(case, seed):
    """From the inputs alone, row group after row group, in float64."""
    s = _inputs(case, seed)
    kind, x = case["kind"], s["x"]
    power_of_two = lambda t: ((t.to(torch.int64) + 1023) << 52).view(torch.float64)
    if kind == "pack":
        b = _blocks(x).double()
        least, last = -126, (10 if x.dtype == torch.float16 else 122)
        top = b.abs().amax(2, keepdim=True)
        t = torch.floor(torch.log2(top.clamp_min(2.0 ** -140))) - 8
        for _ in range(4):                       # the smallest exponent at which the largest value takes at most 127 steps
            t = torch.where(torch.round(top / power_of_two(t)) > 127, t + 1, t)
        t = t.clamp_min(least)
        steps = torch.round(b / power_of_two(t))
        most = torch.where(t == last, 63.0, 127.0)
        back = torch.minimum(torch.maximum(steps, -most), most) * power_of_two(t)
        n, width = x.shape
        return {"back": back.view(n, -1)[:, :width], "masks": x.double() > 0}
    ends, wide = s["ends"], lambda t: t.to(torch.float64)
    n, groups = x.shape[0], case["groups"]
    f64 = dict(dtype=torch.float64, device="cuda")
    if kind.endswith("fwd"):
        y, u = torch.zeros(n, case["outer"], **f64), None
        if kind == "adapter_fwd":
            u = torch.zeros(n, case["rank"], **f64)
        for g in range(groups):
            rows = slice(ends[g], ends[g + 1])
            xs = wide(x[rows])
            if kind == "grouped_fwd":
                y[rows] = torch.matmul(wide(s["W"][g]), xs.t().contiguous()).t()
                continue
            y[rows] = torch.matmul(wide(s["W"]), xs.t().contiguous()).t()
            slot = s["slot_list"][g]
            if slot >= 0:
                u[rows] = wide(s["scales"][slot]) * torch.matmul(wide(s["A"][slot]), xs.t().contiguous()).t()
                y[rows] += torch.matmul(wide(s["B"][slot]), u[rows].t().contiguous()).t()
        if case.get("relu"):
            y = torch.where(y > 0, y, torch.zeros_like(y))
        return {"y": y} if u is None else {"y": y, "u": u}
    if case.get("packed"):
        q, e = s["packed"]
        step = power_of_two(e.to(torch.int64) - 127).repeat_interleave(32, dim=1)
        kept = (q.double() * step)[:, :case["inner"]]
    else:
        kept = wide(x)
    dx = torch.zeros(n, case["inner"], **f64)
    out = {"dx": dx}
    if kind == "grouped_bwd":
        out["dW"] = torch.zeros(s["W"].shape, **f64)
    else:
        out["dA"], out["dB"] = torch.zeros(s["A"].shape, **f64), torch.zeros(s["B"].shape, **f64)
    for g in range(groups):
        rows = slice(ends[g], ends[g + 1])
        d, k = wide(s["dy"][rows]), kept[rows]
        if kind == "grouped_bwd":
            dx[rows] = torch.matmul(d, wide(s["W"][g]))
            out["dW"][g] = torch.matmul(d.t().contiguous(), k)
            continue
        dx[rows] = torch.matmul(d, wide(s["W"]))
        slot = s["slot_list"][g]
        if slot >= 0:
            v = wide(s["scales"][slot]) * torch.matmul(d, wide(s["B"][slot]))
            dx[rows] += torch.matmul(v, wide(s["A"][slot]))
            out["dA"][slot] += torch.matmul(v.t().contiguous(), k)
            out["dB"][slot] += torch.matmul(d.t().contiguous(), wide(s["u"][rows]))
    if case.get("masks"):
        dx[~(x > 0)] = 0.0
    return out


def work(case):
    """Each input read once, each output written once, what is kept between two calls written and read once."""
    b = 4 if case["dtype"] == "f32" else 2
    n, inner = case["n"], case["inner"]
    kind, blocks = case["kind"], (inner + 31) // 32
    if kind == "pack":
        return {"bytes": 2 * n * inner * b + 2 * n * blocks * 33 + 4 * n * blocks + n * inner, "flops": 4 * n * inner}
    outer, groups = case["outer"], case["groups"]
    filled = min(groups - case.get("empty", 0), n)
    kept = n * blocks * 33 if case.get("packed") else n * inner * b
    kept += n * blocks * 4 if case.get("masks") else 0
    if kind == "grouped_fwd":
        return {"bytes": b * (n * (inner + outer) + filled * inner * outer), "flops": 2 * n * inner * outer}
    if kind == "grouped_bwd":
        return {"bytes": kept + b * (n * (inner + outer) + filled * inner * outer) + 4 * groups * inner * outer,
                "flops": 4 * n * inner * outer}
    rank, used = case["rank"], min(case["slots"], filled)
    bank = used * rank * (inner + outer)
    if kind == "adapter_fwd":
        return {"bytes": b * (n * (inner + outer) + inner * outer + bank) + 4 * n * rank,
                "flops": 2 * n * (inner * outer + rank * (inner + outer))}
    return {"bytes": kept + b * (n * (inner + outer) + inner * outer + bank) + 4 * n * rank + 4 * case["slots"] * rank * (inner + outer),
            "flops": 2 * n * (inner * outer + 2 * rank * (inner + outer))}
