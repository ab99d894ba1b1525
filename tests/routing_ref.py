"""Routing to experts and rows kept in 8 bits, stated plainly in 64 bits on the CPU."""
import math

import numpy as np
import torch

import layers_ref as ref

BLOCK = 128
INF = float("inf")


def scores(l, score):
    """[N, E] in 64 bits; 0 where the logit is -inf."""
    l = l.double()
    masked = l == -INF
    if score == "sigmoid":
        s = 1 / (1 + torch.exp(-l))
    else:
        e = torch.where(masked, 0.0, torch.exp(l - l.amax(1, keepdim=True)))
        s = e / e.sum(1, keepdim=True)
    return torch.where(masked, 0.0, s)


def rank(value):
    """Sorted by value, the largest first: a NaN above every number."""
    return (1, 0.0) if math.isnan(value) else (0, value)


def route(logits, topk, score="softmax", bias=None, groups=1, groups_kept=1, group_best=2, renormalise=True, scale=1.0):
    """(ids, weights, scores, load), row by row."""
    l, s = ref.d(logits), scores(ref.d(logits), score)
    N, E = l.shape
    b = [0.0] * E if bias is None else ref.d(bias).tolist()
    ids, weights, load = [], [], [0] * E
    for n in range(N):
        row, sn = l[n].tolist(), s[n].tolist()
        c = [sn[e] + b[e] for e in range(E)]
        can = [e for e in range(E) if row[e] != -INF and c[e] != -INF]
        size = E // groups
        if groups > 1:
            value = []
            for g in range(groups):
                best = sorted((c[e] for e in can if e // size == g), key=rank, reverse=True)[:group_best]
                value.append(sum(best) if best else -INF)
            kept = sorted(range(groups), key=lambda g: rank(value[g]), reverse=True)[:groups_kept]     # (stable: the lower group on a tie)
            can = [e for e in can if e // size in kept]
        chosen = sorted(can, key=lambda e: rank(c[e]), reverse=True)[:topk]
        w = [sn[e] for e in chosen]
        if renormalise:
            total = sum(w)
            w = [0.0 if total == 0 else x / total for x in w]
        for e in chosen:
            load[e] += 1
        ids.append(chosen + [-1] * (topk - len(chosen)))
        weights.append([x * scale for x in w] + [0.0] * (topk - len(chosen)))
    return torch.tensor(ids).reshape(N, topk), torch.tensor(weights, dtype=torch.float64).reshape(N, topk), s, torch.tensor(load)


def weights_of(l, ids, score, renormalise, scale):
    """The weights of held choices, differentiable in l (no row of zero scores)."""
    s = torch.sigmoid(l) if score == "sigmoid" else torch.softmax(l, 1)
    live = (ids >= 0) & (ids < l.shape[1])
    w = s.gather(1, torch.where(live, ids, 0).long()) * live
    if renormalise:
        total = w.sum(1, keepdim=True)
        w = w / torch.where(total > 0, total, 1.0)
    return w * scale, s


def keep(x, code):
    """(codes as numbers, scale as float32) of the rows of x; NaN scales for blocks that are not finite."""
    x = x.detach().cpu().float().numpy()
    N, H = x.shape
    top = ref.TOP[code]
    codes, scale = np.zeros((N, H), np.float32), np.zeros((N, -(-H // BLOCK)), np.float32)
    for b in range(scale.shape[1]):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        m = np.maximum(np.abs(part).max(1, initial=0.0), np.float32(2.0 ** -100))
        with np.errstate(all="ignore"):
            q = (part.astype(np.float64) * top / m[:, None].astype(np.float64)).astype(np.float32)
            scale[:, b] = np.where(np.isfinite(m), m / np.float32(top), np.nan)
        q[~np.isfinite(m)] = 0
        if code == torch.int8:
            codes[:, b * BLOCK:(b + 1) * BLOCK] = np.rint(q)
        else:
            codes[:, b * BLOCK:(b + 1) * BLOCK] = torch.from_numpy(q).to(code).float().numpy()
    return torch.from_numpy(codes), torch.from_numpy(scale)


def stands_for(codes, scale):
    """What codes and scales stand for."""
    codes, scale = codes.detach().cpu().float().double(), scale.detach().cpu().double()
    return codes * scale.repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]
