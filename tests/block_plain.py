"""Plain forms in 64 bits of the operators of a model's block, in numpy, and what
their tests share."""
import numpy as np

U = 2.0 ** -24
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}     # half a step relative to a value
DEV = "cuda"


def say(*a):
    print(*a, flush=True)


def dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def strided(x, gap, shift, dtype):
    """x on the GPU as columns of a wider matrix (gap columns after them, shift elements before the first), the rest
    filled with 77; the matrix and all of its memory."""
    import torch
    n, d = x.shape
    buf = torch.full((n * (d + gap) + shift + 8,), 77.0, dtype=dtype, device=DEV)
    view = buf[shift:shift + n * (d + gap)].view(n, d + gap)[:, :d] if n else buf[:0].view(0, d)
    view.copy_(torch.as_tensor(x).to(DEV))
    return view, buf


def untouched(view, buf, gap, shift):
    """Whether nothing but the matrix was written."""
    import torch
    n, d = view.shape
    keep = torch.ones_like(buf, dtype=torch.bool)
    if n:
        keep[shift:shift + n * (d + gap)].view(n, d + gap)[:, :d] = False
    return bool((buf[keep] == 77).all())


def host(t):
    return t.detach().cpu().double().numpy()


def within(got, want, bound, what):
    """|got - want| <= bound everywhere; tells the worst place."""
    got = host(got) if hasattr(got, "cpu") else got
    off = np.abs(got - want)
    bad = ~(off <= bound)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, off / np.maximum(bound, 1e-300), 0)), off.shape)
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} off, worst at {i}: {got[i]!r}, {want[i]!r} wanted, "
                             f"{off[i]:.3g} of {np.broadcast_to(bound, off.shape)[i]:.3g}")


# ---------------------------------------------------------------- dropout, norm

def kept(rows, dim, drop, seed, first_row=0):
    """Which values dropout keeps."""
    with np.errstate(over="ignore"):
        def mix(z):
            z = (z ^ (z >> np.uint64(30))) * np.uint64(0xbf58476d1ce4e5b9)
            z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94d049bb133111eb)
            return z ^ (z >> np.uint64(31))

        g = np.uint64(0x9e3779b97f4a7c15)
        per = (dim + 3) // 4
        k = (np.uint64(first_row) + np.arange(rows, dtype=np.uint64))[:, None] * np.uint64(per) \
            + np.arange(per, dtype=np.uint64)
        z = mix(mix(np.array(seed % (1 << 64), dtype=np.uint64) + g) + (k + np.uint64(1)) * g)
    bits = np.stack([(z >> np.uint64(16 * i)) & np.uint64(0xffff) for i in range(4)], 2).reshape(rows, 4 * per)
    return bits[:, :dim] >= np.uint64(round(drop * 65536))


def keep_scale(drop):
    return 65536 / (65536 - round(drop * 65536))


def dropped(x, drop, seed, first_row=0):
    if round(drop * 65536) == 0:
        return x
    return np.where(kept(*x.shape, drop, seed, first_row), x * keep_scale(drop), 0.0)


def norm_parts(total, weight, eps, dy):
    """1 / root, n, dtotal without what arrives, and the magnitudes that its rounding errors follow."""
    inv = 1 / np.sqrt((total * total).mean(1, keepdims=True) + eps)
    n = total * inv
    gw = dy * weight
    grad = inv * (gw - n * (gw * n).mean(1, keepdims=True))
    size = inv * (np.abs(gw) + np.abs(n) * np.abs(gw * n).mean(1, keepdims=True))
    return inv, n, grad, size


# ---------------------------------------------------------------- linear attention

def linear(offs, q, k, v, decay, scale, first=None):
    """q [n][g][r][dk], k [n][g][dk], v [n][g][dv]: y [n][g][r][dv], the last states and the state after every position."""
    n, g, r, dk = q.shape
    dv, m = v.shape[2], len(offs) - 1
    y, last, every = np.zeros((n, g, r, dv)), np.zeros((m, g, dk, dv)), np.zeros((n, g, dk, dv))
    for i in range(m):
        s = np.zeros((g, dk, dv)) if first is None else first[i].copy()
        for t in range(offs[i], offs[i + 1]):
            s = decay[:, None, None] * s + k[t][:, :, None] * v[t][:, None]
            every[t] = s
            y[t] = scale * (q[t] @ s)
        last[i] = s
    return y, last, every


def linear_back(offs, q, k, v, decay, scale, every, dy, dlast=None):
    """Gradients of q, k, v and the first states."""
    n, g, r, dk = q.shape
    dv, m = v.shape[2], len(offs) - 1
    dq, dkey, dval, dfirst = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros((m, g, dk, dv))
    for i in range(m):
        s = np.zeros((g, dk, dv)) if dlast is None else dlast[i].copy()
        for t in range(offs[i + 1] - 1, offs[i] - 1, -1):
            s = s + scale * np.swapaxes(q[t], 1, 2) @ dy[t]
            dq[t] = scale * (dy[t] @ np.swapaxes(every[t], 1, 2))
            dkey[t] = (s @ v[t][:, :, None])[:, :, 0]
            dval[t] = (k[t][:, None] @ s)[:, 0]
            s = decay[:, None, None] * s
        dfirst[i] = s
    return dq, dkey, dval, dfirst


# ---------------------------------------------------------------- log probabilities

def answers(x, ids, scale, top=0):
    """Log probabilities of the ids, entropies, all log probabilities, and the top columns of rows of logits."""
    z = x * scale
    with np.errstate(invalid="ignore", divide="ignore"):
        most = z.max(1, keepdims=True)
        log = most + np.log(np.exp(z - most).sum(1, keepdims=True))
        every = z - log
        p = np.exp(every)
        entropy = -np.where(p > 0, p * every, 0.0).sum(1)
    real = (ids >= 0) & (ids < x.shape[1])
    logp = np.where(real, every[np.arange(len(ids)), np.where(real, ids, 0)], 0.0)
    order = np.argsort(-x, axis=1, kind="stable")[:, :top]
    return logp, entropy, every, order


def answers_back(every, ids, entropy, scale, dlogp, dentropy=None):
    """Gradient of the logits."""
    p = np.exp(every)
    real = (ids >= 0) & (ids < every.shape[1])
    dl = np.where(real, dlogp, 0.0)
    dx = -dl[:, None] * p
    dx[np.arange(len(ids))[real], ids[real]] += dl[real]
    if dentropy is not None:
        dx -= dentropy[:, None] * p * (np.where(p > 0, every, 0.0) + entropy[:, None])
    return scale * dx
