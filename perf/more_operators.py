"""Routing to experts and 8-bit activation checkpoints, around the 2:4 products of a feed-forward block: listed cases, and draws from the same ranges.

Five kinds, each as a program makes the calls:

``route``         the router's logits to the experts of every token and their weights: softmax or sigmoid scores, a bias for balance, groups
``route_grad``    from the gradient of those weights (and of the scores) back to the logits
``keep``          rows kept in 8 bits with a scale for every 128 values, and had again: through the activation, or in the experts' order
``layer_grad``    the gradients of a layer whose rows, in front and behind, were kept so: through the activation, of the bias and of the weights
``experts_grad``  the same of every expert, its rows taken from the tokens' kept ones

Sizes are those of this repository's workloads, tests and measured tables, or generic layer sizes.
"""
import math

import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "i8": torch.int8, "f8": torch.float8_e4m3fn}
_SIZE = {"f16": 2, "bf16": 2, "f32": 4}
_TOP = {"i8": 127.0, "f8": 448.0}
_BLOCK = 128                    # neighbouring values of a row under one scale
_ROWS = 16                      # segments of sorted rows begin at multiples of this


def listed():
    return [
        # decoding: one token of each of 16 sequences to four of 64 experts; the launch is all there is
        dict(name="route_decode", kind="route", N=16, E=64, topk=4, dtype="f32", score="softmax", bias=False, groups=1, kept=1, best=1,
             renormalise=True, scale=1.0, scores=False, load=False),
        # a batch of 16 x 512 tokens to eight of 256 experts out of four of eight groups, with the balance bias and the load that it follows
        dict(name="route_groups", kind="route", N=8192, E=256, topk=8, dtype="f32", score="sigmoid", bias=True, groups=8, kept=4, best=2,
             renormalise=True, scale=2.5, scores=False, load=True),
        # a fine-tuning step on a prompt of arbitrary length, two of eight experts
        dict(name="route_grad_prompt", kind="route_grad", N=509, E=8, topk=2, dtype="bf16", score="softmax", renormalise=True, scale=1.0, scores=False,
             dropped=0.0),
        # a training batch with a balance loss on the scores, one token in twenty without some of its experts
        dict(name="route_grad_balance", kind="route_grad", N=8192, E=256, topk=8, dtype="f32", score="softmax", renormalise=False, scale=1.0, scores=True,
             dropped=0.05),
        # a short prompt, rows of no whole blocks
        dict(name="keep_prompt", kind="keep", N=509, H=1000, dtype="f16", code="i8", act="none", topk=0, E=0),
        # a training batch's rows in front of a wide layer
        dict(name="keep_batch", kind="keep", N=8192, H=4096, dtype="bf16", code="i8", act="none", topk=0, E=0),
        # the rows behind an up-projection, activated again for the next layer's gradient
        dict(name="keep_gelu", kind="keep", N=4096, H=4096, dtype="bf16", code="f8", act="gelu", topk=0, E=0),
        # tokens kept once, and had in the order of their two of eight experts
        dict(name="keep_experts", kind="keep", N=4096, H=1024, dtype="bf16", code="i8", act="none", topk=2, E=8),
        # a layer of odd sizes on a prompt of arbitrary length
        dict(name="layer_grad_prompt", kind="layer_grad", M=640, K=1000, N=509, dtype="f16", code="f8", act="silu"),
        # the up-projection of a block on a training batch
        dict(name="layer_grad_batch", kind="layer_grad", M=4096, K=1024, N=8192, dtype="bf16", code="i8", act="gelu"),
        # four small experts on a few tokens
        dict(name="experts_grad_few", kind="experts_grad", N=37, topk=2, E=4, M=256, K=264, dtype="bf16", code="f8", act="silu"),
        # eight experts on a training batch
        dict(name="experts_grad_batch", kind="experts_grad", N=4096, topk=2, E=8, M=2048, K=1024, dtype="bf16", code="i8", act="silu"),
    ]


# ---- draws -----------------------------------------------------------------------------------------------------

def _size(rng, lo, hi, multiple=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(int(round(v / multiple)), -(-lo // multiple)) * multiple


def _draw_experts_number(rng):
    return rng.choice([8, 16, 64, 128, 256, rng.randint(2, 256), _size(rng, 2, 1024)])


def _draw_route(rng):
    E, N = _draw_experts_number(rng), _size(rng, 1, 16384)
    while N * E > 1 << 21:
        N = max(1, N // 2)
    groups = rng.choice([1, 1] + [g for g in (2, 4, 8) if E % g == 0])
    kept = rng.randint(1, groups)
    topk = min(kept * (E // groups), rng.choice([1, 2, 2, 4, 6, 8, 8, rng.randint(1, 16)]))
    return dict(kind="route", N=N, E=E, topk=topk, dtype=rng.choice(["f32", "f32", "bf16", "f16"]), score=rng.choice(["softmax", "sigmoid"]),
                bias=rng.random() < 0.5, groups=groups, kept=kept, best=rng.choice([1, 2]), renormalise=rng.random() < 0.6,
                scale=rng.choice([1.0, 2.5]), scores=rng.random() < 0.3, load=rng.random() < 0.4)


def _draw_route_grad(rng):
    E, N = _draw_experts_number(rng), _size(rng, 1, 16384)
    while N * E > 1 << 21:
        N = max(1, N // 2)
    return dict(kind="route_grad", N=N, E=E, topk=min(E, rng.choice([1, 2, 2, 4, 6, 8, 8, rng.randint(1, 16)])), dtype=rng.choice(["f32", "f32", "bf16", "f16"]),
                score=rng.choice(["softmax", "sigmoid"]), renormalise=rng.random() < 0.6, scale=rng.choice([1.0, 2.5]), scores=rng.random() < 0.4,
                dropped=rng.choice([0.0, 0.0, 0.1]))


def _draw_keep(rng):
    N, H = _size(rng, 1, 16384), _size(rng, 32, 16384, rng.choice([128, 64, 8, 1]))
    E = rng.choice([0, 0, 4, 8, 64])
    topk = min(E, rng.choice([1, 2, 2, 4]))
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    while N * max(topk, 1) * H * _SIZE[dtype] > 1 << 26:
        N = max(1, N // 2)
    return dict(kind="keep", N=N, H=H, dtype=dtype, code=rng.choice(["i8", "i8", "f8"]),
                act=rng.choice(["none", "none", "relu", "gelu", "silu"]), topk=topk, E=E)


def _draw_layer_grad(rng):
    M, K, N = _size(rng, 128, 8192, rng.choice([64, 64, 8, 1])), _size(rng, 128, 8192, rng.choice([64, 64, 8, 1])), _size(rng, 1, 16384)
    while M * K * N > 1 << 35:
        N = max(1, N // 2)
    while M * K > 1 << 24:
        M, K = max(128, M // 2), max(128, K // 2)
    return dict(kind="layer_grad", M=M, K=K, N=N, dtype=rng.choice(["bf16", "bf16", "f16"]), code=rng.choice(["i8", "i8", "f8"]),
                act=rng.choice(["none", "relu", "gelu", "silu"]))


def _draw_experts_grad(rng):
    E = rng.choice([4, 8, 8, 16, 32])
    topk, N = min(E, rng.choice([1, 2, 2, 4])), _size(rng, 1, 4096)
    M, K = _size(rng, 128, 4096, 64), _size(rng, 128, 4096, rng.choice([64, 64, 8]))
    while E * M * K > 1 << 25:
        M, K = max(128, M // 2), max(128, K // 2 // 8 * 8)
    while N * topk * M * K > 1 << 34:
        N = max(1, N // 2)
    return dict(kind="experts_grad", N=N, topk=topk, E=E, M=M, K=K, dtype=rng.choice(["bf16", "bf16", "f16"]), code=rng.choice(["i8", "i8", "f8"]),
                act=rng.choice(["none", "relu", "gelu", "silu"]))


def draw(rng):
    return rng.choice([_draw_route] * 4 + [_draw_route_grad] * 3 + [_draw_keep] * 4 + [_draw_layer_grad] * 4 + [_draw_experts_grad] * 3)(rng)


# ---- what a program has in hand before the call ----------------------------------------------------------------

def _logits(g, N, E, dtype):
    """A router's logits, some experts more popular than others."""
    return (torch.randn(N, E, generator=g, device="cuda") + 0.5 * torch.randn(E, generator=g, device="cuda")).to(_TYPES[dtype])


def _activations(g, N, H, dtype):
    """Rows of unit variance with a few channels far larger than the others, as a residual stream has them."""
    x = torch.randn(N, H, generator=g, device="cuda")
    loud = torch.rand(H, generator=g, device="cuda") < 0.01
    return (x * torch.where(loud, 20.0, 1.0)).to(_TYPES[dtype])


def _blocks(x):
    """[N, blocks, 128] of the rows of x, zeros behind their end."""
    pad = -x.shape[1] % _BLOCK
    return torch.nn.functional.pad(x, (0, pad)).view(x.shape[0], -1, _BLOCK)


def _kept(x, code):
    """(codes, scale): the rows of x in 8 bits.  The quotient is taken in 64 bits, where no code is next to a border by accident."""
    b = _blocks(x.double())
    most = b.abs().amax(2).clamp(min=2.0 ** -100)
    q = (b * _TOP[code] / most[..., None]).float()
    q = q.round().to(torch.int8) if code == "i8" else q.to(torch.float8_e4m3fn)
    scale = most.float() / torch.full_like(most, _TOP[code], dtype=torch.float32)
    raw = q.view(torch.int8).reshape(x.shape[0], -1)[:, :x.shape[1]].contiguous()
    return raw.view(_TYPES[code]), scale


def _had(codes, scale, wide=torch.float32):
    """What kept rows stand for."""
    return codes.to(torch.float32).to(wide) * scale.to(wide).repeat_interleave(_BLOCK, dim=1)[:, :codes.shape[1]]


def _choices(g, N, topk, E):
    return (torch.randn(N, E, generator=g, device="cuda") + torch.randn(E, generator=g, device="cuda")).topk(topk, dim=1).indices.to(torch.int32)


def _sorted(ids, E):
    """offsets [E + 1] and rows [R] of the choices in order of their expert: the segment of expert e is rows offsets[e] .. offsets[e+1] - 1,
    whole sixteens; row: its choice n * k + j, or -1."""
    flat = ids.reshape(-1).long()
    T = flat.numel()
    count = torch.zeros(E, dtype=torch.int64, device=ids.device).scatter_add_(0, flat, torch.ones_like(flat))
    starts = count.cumsum(0) - count
    padded = (count + _ROWS - 1) // _ROWS * _ROWS
    offsets = torch.cat([padded.new_zeros(1), padded.cumsum(0)])
    order = torch.argsort(flat, stable=True)
    at = flat[order]
    rows = torch.full(((T + (_ROWS - 1) * min(T, E)) // _ROWS * _ROWS,), -1, dtype=torch.int64, device=ids.device)
    rows[offsets[at] + torch.arange(T, device=ids.device) - starts[at]] = order
    return offsets.to(torch.int32), rows.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    kind, N, dtype = case["kind"], case["N"], case["dtype"]
    if kind == "route":
        s["logits"] = _logits(g, N, case["E"], dtype)
        s["b"] = 0.05 * torch.randn(case["E"], generator=g, device="cuda") if case["bias"] else None
    elif kind == "route_grad":
        s["logits"] = _logits(g, N, case["E"], dtype)
        s["ids"] = s["logits"].float().topk(case["topk"], dim=1).indices.to(torch.int32)
        if case["dropped"]:
            s["ids"] = torch.where(torch.rand(N, case["topk"], generator=g, device="cuda") < case["dropped"], -1, s["ids"])
        s["dw"] = 0.1 * torch.randn(N, case["topk"], generator=g, device="cuda")
        s["ds"] = 0.01 * torch.randn(N, case["E"], generator=g, device="cuda") if case["scores"] else None
    elif kind == "keep":
        s["x"] = _activations(g, N, case["H"], dtype)
        s["rows"] = _sorted(_choices(g, N, case["topk"], case["E"]), case["E"])[1] if case["topk"] else None
    else:
        s["x"] = _kept(_activations(g, N, case["K"], dtype), case["code"])
        R = N
        if kind == "experts_grad":
            s["offsets"], s["rows"] = _sorted(_choices(g, N, case["topk"], case["E"]), case["E"])
            R = s["rows"].numel()
        z, dy = torch.randn(R, case["M"], generator=g, device="cuda"), 0.1 * torch.randn(R, case["M"], generator=g, device="cuda")
        if kind == "experts_grad":
            live = (s["rows"] >= 0)[:, None]
            z, dy = torch.where(live, z, 0), torch.where(live, dy, 0)
        s["dy"] = dy.to(_TYPES[dtype])
        s["z"] = _kept(z.to(_TYPES[dtype]), case["code"]) if case["act"] != "none" else None
    return s


# ---- one pass, in plain form -----------------------------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    p = torch.sigmoid(z)
    return p * (1 + z * (1 - p))


def _scores(l, score):
    """In 64 bits: two experts' scores are often closer than 32 bits tell apart."""
    l = l.double()
    if score == "sigmoid":
        return 1 / (1 + torch.exp(-l))
    e = torch.exp(l - l.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain_route(s):
    E, groups = s["E"], s["groups"]
    score = _scores(s["logits"], s["score"])
    choice = score if s["b"] is None else score + s["b"].double()
    if groups > 1:
        value = choice.view(-1, groups, E // groups).sort(dim=2, descending=True).values[..., :s["best"]].sum(2)
        best = value.sort(dim=1, descending=True, stable=True).indices[:, :s["kept"]]
        stays = torch.zeros_like(value, dtype=torch.bool).scatter_(1, best, True)
        choice = torch.where(stays.repeat_interleave(E // groups, dim=1), choice, -math.inf)
    ids = choice.sort(dim=1, descending=True, stable=True).indices[:, :s["topk"]]
    w = score.gather(1, ids)
    if s["renormalise"]:
        w = w / w.sum(1, keepdim=True)
    got = {"ids": ids.to(torch.int32), "weights": (w * s["scale"]).float()}
    if s["scores"]:
        got["scores"] = score.float()
    if s["load"]:
        flat = ids.reshape(-1)
        got["load"] = torch.zeros(E, dtype=torch.int64, device=flat.device).scatter_add_(0, flat, torch.ones_like(flat)).to(torch.int32)
    return got


def _plain_route_grad(s):
    score, live, dw = _scores(s["logits"], s["score"]), s["ids"] >= 0, s["dw"].double()
    at = s["ids"].long().clamp(min=0)
    if s["renormalise"]:
        w = torch.where(live, score.gather(1, at), 0)
        total = w.sum(1, keepdim=True)
        dw = (dw - (dw * w).sum(1, keepdim=True) / total) / total
    g = (torch.zeros_like(score) if s["ds"] is None else s["ds"].double()).scatter_add(1, at, torch.where(live, dw * s["scale"], 0))
    d = score * (1 - score) * g if s["score"] == "sigmoid" else score * (g - (g * score).sum(1, keepdim=True))
    return {"dlogits": torch.where(score > 0, d, 0).to(s["logits"].dtype)}


def _gathered(x, rows, topk):
    return torch.where(rows[:, None] >= 0, x[(rows.long() // topk).clamp(min=0)], 0)


def _plain(s):
    kind = s["kind"]
    if kind == "route":
        return _plain_route(s)
    if kind == "route_grad":
        return _plain_route_grad(s)
    out = _TYPES[s["dtype"]]
    if kind == "keep":
        codes, scale = _kept(s["x"], s["code"])
        y = _act(_had(codes, scale), s["act"])
        return {"scale": scale, "y": (y if s["rows"] is None else _gathered(y, s["rows"], s["topk"])).to(out)}
    dz = s["dy"].float()
    if s["z"] is not None:
        dz = dz * _act_slope(_had(*s["z"]), s["act"])
    x = _had(*s["x"])
    if kind == "layer_grad":
        return {"dz": dz.to(out), "db": dz.sum(0), "dW": (dz.t() @ x).to(out)}
    E, o = s["E"], s["offsets"].long()
    x = _gathered(x, s["rows"], s["topk"])
    at = torch.arange(max(int((o[1:] - o[:-1]).max()), 1), device=o.device)             # [E, C]: the rows of every segment
    there, rows = at < (o[1:] - o[:-1])[:, None], (o[:-1, None] + at).clamp(max=x.shape[0] - 1)
    live = torch.where(there[..., None], dz[rows], 0)
    return {"dz": dz.to(out), "db": live.sum(1), "dW": torch.bmm(live.transpose(1, 2).contiguous(), x[rows]).to(out)}


# ---- one pass --------------------------------------------------------------------------------------------------

def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2104_08378_amd import sp24
    kind, dtype = s["kind"], _TYPES[s["dtype"]]
    if kind == "route":
        r = sp24.sp24_moe_route(s["logits"], s["topk"], score=s["score"], bias=s["b"], groups=s["groups"], groups_kept=s["kept"], group_best=s["best"],
                                renormalise=s["renormalise"], scale=s["scale"], want_scores=s["scores"], want_load=s["load"])
        got = {"ids": r.ids, "weights": r.weights}
        if s["scores"]:
            got["scores"] = r.scores
        if s["load"]:
            got["load"] = r.load
        return got
    if kind == "route_grad":
        return {"dlogits": sp24.sp24_moe_route_backward(s["logits"], s["ids"], s["dw"], score=s["score"], renormalise=s["renormalise"], scale=s["scale"],
                                                        dscores=s["ds"])}
    if kind == "keep":
        kept = sp24.sp24_checkpoint_rows(s["x"], _TYPES[s["code"]])
        return {"scale": kept.scale, "y": sp24.sp24_restore_rows(kept, dtype, act=s["act"], rows=s["rows"], topk=max(s["topk"], 1))}
    x, z = (None if k is None else sp24.Checkpoint(*k) for k in (s["x"], s["z"]))
    if kind == "layer_grad":
        dz, dzt, db = sp24.sp24_linear_backward_checkpoint(s["dy"], z, s["act"])
        return {"dz": dz, "db": db, "dW": sp24.sp24_gemm_dense_checkpoint(dzt, x, dtype)}
    dz, dzt, db = sp24.sp24_linear_backward_checkpoint(s["dy"], z, s["act"], offsets=s["offsets"])
    return {"dz": dz, "db": db, "dW": sp24.sp24_gemm_dense_grouped_checkpoint(dzt, x, s["offsets"], dtype, rows=s["rows"], topk=s["topk"])}


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def _kept_bytes(N, H):
    return N * (H + 4 * -(-H // _BLOCK))


def work(case):
    """Bytes: every input read once, every output written once.  A kept form that the pass itself makes and reads counts once."""
    kind, N, es = case["kind"], case["N"], _SIZE[case["dtype"]]
    if kind == "route":
        E, T = case["E"], N * case["topk"]
        return {"bytes": N * E * (es + 4 * case["scores"]) + 8 * T + 4 * E * (case["bias"] + case["load"]), "flops": 10 * N * E}
    if kind == "route_grad":
        E, T = case["E"], N * case["topk"]
        return {"bytes": N * E * (2 * es + 4 * case["scores"]) + 8 * T, "flops": 12 * N * E}
    if kind == "keep":
        T = N * max(case["topk"], 1)
        return {"bytes": N * case["H"] * es + _kept_bytes(N, case["H"]) + T * case["H"] * es, "flops": 8 * (N + T) * case["H"]}
    M, K, T = case["M"], case["K"], N * case.get("topk", 1)
    return {"bytes": _kept_bytes(N, K) + (_kept_bytes(T, M) if case["act"] != "none" else 0) + es * (2 * T * M + case.get("E", 1) * M * K),
            "flops": 2 * T * M * K}


# ---- the same in 64 bits ---------------------------------------------------------------------------------------

def _value64(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))      # 1 + tanh u = 2 sigmoid 2u
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z * 1


def _slope64(z, act):
    """The activation's derivative, taken by automatic differentiation of its formula."""
    z = z.clone().requires_grad_(True)
    with torch.enable_grad():
        y = _value64(z, act).sum()
    return torch.autograd.grad(y, z)[0]


def _stands_for64(kept):
    codes, scale = kept
    out = torch.empty(codes.shape, dtype=torch.float64, device=codes.device)
    for b in range(scale.shape[1]):
        part = slice(b * _BLOCK, (b + 1) * _BLOCK)
        out[:, part] = codes[:, part].float().double() * scale[:, b, None].double()
    return out


def _keep64(x, code):
    """(scale, what the codes stand for)"""
    x = x.double()
    scale, out = [], torch.empty_like(x)
    for first in range(0, x.shape[1], _BLOCK):
        part = x[:, first:first + _BLOCK]
        unit = part.abs().max(1).values.clamp(min=2.0 ** -100)
        scale.append(unit / _TOP[code])
        q = part * _TOP[code] / unit[:, None]
        step = 1.0 if code == "i8" else torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)   # of 3 fraction bits, exponents from -6 on
        out[:, first:first + _BLOCK] = torch.round(q / step) * step * scale[-1][:, None]
    return torch.stack(scale, 1), out


def _log_scores64(l, score):
    l = l.double()
    return -torch.nn.functional.softplus(-l) if score == "sigmoid" else torch.log_softmax(l, 1)


def _route64(s):
    import numpy as np
    score = _log_scores64(s["logits"], s["score"]).exp().cpu().numpy()
    choice = score + (0 if s["b"] is None else s["b"].double().cpu().numpy())
    N, E = score.shape
    order = np.argsort(-choice, axis=1, kind="stable")
    if s["groups"] > 1:
        size = E // s["groups"]
        value = np.stack([np.sort(choice[:, i * size:(i + 1) * size], axis=1)[:, ::-1][:, :s["best"]].sum(1) for i in range(s["groups"])], 1)
        rank = np.argsort(np.argsort(-value, axis=1, kind="stable"), axis=1)
        out = (rank >= s["kept"])[np.arange(N)[:, None], order // size]                 # of a group that does not stay: behind all others
        order = np.take_along_axis(order, np.argsort(out, axis=1, kind="stable"), 1)
    ids = order[:, :s["topk"]]
    w = np.take_along_axis(score, ids, 1)
    w = s["scale"] * (w / w.sum(1, keepdims=True) if s["renormalise"] else w)
    tensor = lambda v, t: torch.from_numpy(np.ascontiguousarray(v)).to(t).cuda()  # noqa: E731
    got = {"ids": tensor(ids, torch.int32), "weights": tensor(w, torch.float64)}
    if s["scores"]:
        got["scores"] = tensor(score, torch.float64)
    if s["load"]:
        got["load"] = tensor(np.bincount(ids.reshape(-1), minlength=E), torch.int32)
    return got


def _route_grad64(s):
    """By automatic differentiation of the weights and scores in 64 bits."""
    l = s["logits"].double().requires_grad_(True)
    with torch.enable_grad():
        score = _log_scores64(l, s["score"]).exp()
        w = score.gather(1, s["ids"].long().clamp(min=0)) * (s["ids"] >= 0)
        if s["renormalise"]:
            total = w.sum(1, keepdim=True)
            w = w / torch.where(total > 0, total, 1)
        loss = (w * s["scale"] * s["dw"].double()).sum()
        if s["ds"] is not None:
            loss = loss + (score * s["ds"].double()).sum()
    return {"dlogits": torch.autograd.grad(loss, l)[0]}


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "route":
        return _route64(s)
    if kind == "route_grad":
        return _route_grad64(s)
    if kind == "keep":
        scale, y = _keep64(s["x"], s["code"])
        y = _value64(y, s["act"])
        if s["rows"] is None:
            return {"scale": scale, "y": y}
        out, live = torch.zeros(s["rows"].numel(), y.shape[1], dtype=torch.float64, device=y.device), s["rows"] >= 0
        out[live] = y[s["rows"][live].long() // s["topk"]]
        return {"scale": scale, "y": out}
    dz = s["dy"].double()
    if s["z"] is not None:
        dz = dz * _slope64(_stands_for64(s["z"]), s["act"])
    x = _stands_for64(s["x"])
    if kind == "layer_grad":
        return {"dz": dz, "db": dz.sum(0), "dW": dz.t() @ x}
    o, rows = s["offsets"].cpu().tolist(), s["rows"].long()
    db, dW = dz.new_zeros(s["E"], s["M"]), dz.new_zeros(s["E"], s["M"], s["K"])
    for e in range(s["E"]):
        part = dz[o[e]:o[e + 1]]
        at = rows[o[e]:o[e + 1]]
        db[e] = part.sum(0)
        dW[e] = part[at >= 0].t() @ x[at[at >= 0] // s["topk"]]
    return {"dz": dz, "db": db, "dW": dW}
