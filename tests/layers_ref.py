"""The operators around the products, stated plainly in 64 bits on the CPU, and how far a result may be from that."""
import math

import torch

#: half a unit of the last place, relative, and the smallest step's half, for results rounded once
HALF_ULP = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 2.0 ** -134)}
TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def d(t):
    """The values in 64 bits on the CPU."""
    return t.detach().cpu().to(torch.float32).double() if t.element_size() == 1 else t.detach().cpu().double()


def close(got, want, err=0.0, what=""):
    """Every value within one rounding to its type of a number that is at most ``err`` off."""
    half, least = HALF_ULP[got.dtype]
    g = d(got)
    err = torch.as_tensor(err, dtype=torch.float64)
    room = half * (want.abs() + err) + least + err
    same = (g == want) | (torch.isnan(g) & torch.isnan(want))
    bad = ~same & ~((g - want).abs() <= room * 1.0000001)
    assert not bool(bad.any()), (what, int(bad.sum()), float((g - want).abs()[bad].max() if bool((~torch.isnan(g[bad])).any()) else math.nan),
                                 g[bad][:4].tolist(), want[bad][:4].tolist())


def act(z, name):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z.clone()


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def norm(x, w, eps, r=None):
    h = d(x) + (0 if r is None else d(r))
    rstd = 1 / torch.sqrt(h.square().mean(1) + eps)
    return h, rstd, h * rstd[:, None] * d(w)


def norm_grad(dy, h, w, rstd, dh=None):
    dy, h, w, v = d(dy), d(h), d(w), d(rstd)[:, None]
    g = dy * w
    dx = v * (g - h * v * v * (g * h).mean(1, keepdim=True))
    return dx if dh is None else dx + d(dh), (dy * h * v).sum(0)


def sort(ids, experts):
    flat = ids.reshape(-1).tolist()
    members = [[i for i, e in enumerate(flat) if e == x] for x in range(experts)] if experts <= 8 else None
    if members is None:
        members = [[] for _ in range(experts)]
        for i, e in enumerate(flat):
            if 0 <= e < experts:
                members[e].append(i)
    R = (len(flat) + 15 * min(len(flat), experts)) // 16 * 16
    offsets, slots, rows = [0], [-1] * len(flat), [-1] * R
    for m in members:
        for k, i in enumerate(m):
            slots[i], rows[offsets[-1] + k] = offsets[-1] + k, i
        offsets.append(offsets[-1] + -(-len(m) // 16) * 16)
    return offsets, slots, rows


def per_row(offsets, R):
    """The expert of every row, -1 behind the last segment."""
    e = torch.full((R,), -1, dtype=torch.int64)
    for i in range(len(offsets) - 1):
        e[offsets[i]:offsets[i + 1]] = i
    return e
