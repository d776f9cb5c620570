"""Float64 definitions of the layers whose rows choose their matrices: grouped products, low-rank adapters beside a shared
matrix, and layer inputs in 8 bits.  numpy only; shares nothing with the GPU path.

Group g owns rows offsets[g] .. offsets[g+1]-1; rows outside every group come back as NaN ("not written")."""
import numpy as np


def group_ranges(offsets, n, groups):
    if offsets is None:
        return [(0, n)]
    return [(int(offsets[g]), int(offsets[g + 1])) for g in range(groups)]


def relu(z):
    return np.where(z <= 0, 0.0, z)


def grouped_forward(x, W, offsets, use_relu=False):
    x, W = np.asarray(x, np.float64), np.asarray(W, np.float64)
    y = np.full((x.shape[0], W.shape[1]), np.nan)
    for g, (lo, hi) in enumerate(group_ranges(offsets, x.shape[0], W.shape[0])):
        y[lo:hi] = x[lo:hi] @ W[g].T
    return relu(y) if use_relu else y


def grouped_backward(x, W, offsets, dy, mask=None):
    """dx [n, in] (zero where `mask` is false), dW [groups, out, in]."""
    x, W, dy = (np.asarray(t, np.float64) for t in (x, W, dy))
    dx, dW = np.full(x.shape, np.nan), np.zeros(W.shape)
    for g, (lo, hi) in enumerate(group_ranges(offsets, x.shape[0], W.shape[0])):
        dx[lo:hi] = dy[lo:hi] @ W[g]
        dW[g] = dy[lo:hi].T @ x[lo:hi]
    if mask is not None:
        dx = np.where(mask, dx, np.where(np.isnan(dx), dx, 0.0))
    return dx, dW


def _slot(slots, g, adapters):
    s = g if slots is None else int(slots[g])
    return s if 0 <= s < adapters else -1


def adapter_forward(x, W, A, B, scales, slots, offsets, use_relu=False):
    """y [n, out], u [n, rank]."""
    x, W, A, B = (np.asarray(t, np.float64) for t in (x, W, A, B))
    n, groups = x.shape[0], len(offsets) - 1
    y, u = np.full((n, W.shape[0]), np.nan), np.full((n, A.shape[1]), np.nan)
    for g, (lo, hi) in enumerate(group_ranges(offsets, n, groups)):
        s = _slot(slots, g, A.shape[0])
        y[lo:hi] = x[lo:hi] @ W.T
        u[lo:hi] = 0.0
        if s >= 0:
            u[lo:hi] = float(scales[s]) * (x[lo:hi] @ A[s].T)
            y[lo:hi] += u[lo:hi] @ B[s].T
    return (relu(y) if use_relu else y), u


def adapter_backward(x, W, A, B, scales, slots, offsets, u, dy, mask=None):
    """dx [n, in], dA, dB (shaped like the bank)."""
    x, W, A, B, u, dy = (np.asarray(t, np.float64) for t in (x, W, A, B, u, dy))
    n, groups = x.shape[0], len(offsets) - 1
    dx, dA, dB = np.full(x.shape, np.nan), np.zeros(A.shape), np.zeros(B.shape)
    for g, (lo, hi) in enumerate(group_ranges(offsets, n, groups)):
        s = _slot(slots, g, A.shape[0])
        dx[lo:hi] = dy[lo:hi] @ W
        if s >= 0:
            v = float(scales[s]) * (dy[lo:hi] @ B[s])
            dx[lo:hi] += v @ A[s]
            dA[s] += v.T @ x[lo:hi]
            dB[s] += dy[lo:hi].T @ u[lo:hi]
    if mask is not None:
        dx = np.where(mask, dx, np.where(np.isnan(dx), dx, 0.0))
    return dx, dA, dB


LAST_EXPONENT = {"f32": 122, "bf16": 122, "f16": 10}     # beyond 63 steps of this the type has no number


def pack8(x, dtype):
    """q int8 [n, 32 * blocks], e uint8 [n, blocks], mask bool [n, dim]; x holds numbers of `dtype`."""
    x = np.asarray(x, np.float64)
    n, dim = x.shape
    blocks = (dim + 31) // 32
    full = np.zeros((n, 32 * blocks))
    full[:, :dim] = x
    v = full.reshape(n, blocks, 32)
    finite = np.all(np.isfinite(v), axis=2)
    v = np.where(finite[..., None], v, 0.0)
    top = np.max(np.abs(v), axis=2)
    with np.errstate(divide="ignore"):
        t = np.where(top > 0, np.floor(np.log2(top)) - 9, -126.0)
    t = np.maximum(t, -126).astype(np.int64)
    while np.any(np.rint(np.ldexp(top, -t)) > 127):
        t += np.rint(np.ldexp(top, -t)) > 127
    most = np.where(t == LAST_EXPONENT[dtype], 63, 127)[..., None]
    q = np.clip(np.rint(np.ldexp(v, -t[..., None])), -most, most).astype(np.int8).reshape(n, -1)
    e = np.where(finite, t + 127, 255).astype(np.uint8)
    with np.errstate(invalid="ignore"):
        return q, e, x > 0


def unpack8(q, e, dim):
    step = np.where(e == 255, np.nan, np.ldexp(1.0, e.astype(np.int64) - 127))
    return (q.astype(np.float64) * np.repeat(step, 32, axis=1))[:, :dim]


def mask_words(mask):
    """Bit c % 32 of word c / 32, as int32."""
    n, dim = mask.shape
    blocks = (dim + 31) // 32
    full = np.zeros((n, 32 * blocks), np.uint64)
    full[:, :dim] = mask
    return (full.reshape(n, blocks, 32) << np.arange(32, dtype=np.uint64)).sum(axis=2).astype(np.uint32).view(np.int32)
