"""Timing cases of the operators of a decoder layer that stand before the preconditioner: the root-mean-square norm
with the residual's addition, dropout from a counter-based generator, and causal attention over packed sequences,
each with its gradient.  Their products are the weight gradients that the statistics are accumulated from.

A case is a dict of plain values; ``listed()`` holds the fixed ones, ``draw(rng)`` makes one more of the same ranges.
Fields (those of the other kinds are left out of a case):

    kind      "norm" (rms_norm), "norm_grad" (rms_norm_backward), "dropout" (dropout, forward and backward being the same
              call), "attention" (the forward pass), "attention_train" (forward and backward)
    rows, cols  of the matrices of norm and dropout
    x, h, y, w  types of the norm's input (and its gradient), of the residual stream, of the output (its gradient), of
                the weight: "fp32", "bf16"; y also "e4m3", 8 bits with fp32 scales
    group     columns that share a scale (0: the row)
    drop      probability of dropout, a multiple of 2^-16 (0: none)
    lens      lengths of the packed sequences, a text of numbers joined by commas
    tail      rows behind the last sequence, left as they were
    heads, kv_heads, dim, dtype   of the attention
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
E4M3_MAX = 448.0
SCALE_FLOOR = 2.0 ** -100
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
BYTES = {"fp32": 4, "bf16": 2, "e4m3": 1}


def _norm(**kw):
    return {"kind": "norm", "x": "bf16", "h": "bf16", "y": "bf16", "w": "bf16", "group": 0, "drop": 0.0, **kw}


def _attention(**kw):
    return {"kind": "attention", "heads": 32, "kv_heads": 4, "dim": 64, "dtype": "bf16", "tail": 0, **kw}


def listed():
    return [
        # a handful of new rows of the 1.1B model (2048 wide): latency
        _norm(name="norm_few_rows", rows=4, cols=2048),
        # a training batch of it before a product on 8 bits, dropout before the residual, one scale per 128 columns
        _norm(name="norm_batch_e4m3", rows=16384, cols=2048, y="e4m3", group=128, drop=6554 / 65536),
        # rows of no round size of a small fp32 model
        _norm(name="norm_ragged_fp32", rows=1001, cols=777, x="fp32", h="fp32", y="fp32", w="fp32"),
        # gradient of the training batch, the residual stream in fp32, with dropout
        _norm(name="norm_grad_batch", kind="norm_grad", rows=16384, cols=2048, h="fp32", drop=6554 / 65536),
        # gradient at the width of the feed-forward part, a short batch
        _norm(name="norm_grad_wide", kind="norm_grad", rows=600, cols=5632),
        # dropout of a small matrix of no round size
        {"name": "dropout_small_fp32", "kind": "dropout", "rows": 777, "cols": 1001, "x": "fp32", "drop": 0.25},
        # dropout of the hidden activations of a training batch
        {"name": "dropout_batch", "kind": "dropout", "rows": 16384, "cols": 5632, "x": "bf16", "drop": 6554 / 65536},
        # short packed documents, forward only: latency
        _attention(name="attention_short", lens="1,17,64,0,130,31", tail=13),
        # evaluation of one long document of the 1.1B model
        _attention(name="attention_long", lens="8192"),
        # a training batch of it: four documents that fill their context
        _attention(name="attention_train_batch", kind="attention_train", lens="2048,2048,2048,2048"),
        # packed documents of uneven lengths with wide heads, as a data loader without padding gives them
        _attention(name="attention_train_packed", kind="attention_train", lens="3001,257,64,1900,1,777,1023,1100", tail=69, heads=16,
                   kv_heads=4, dim=128),
        # a small fp32 model, every head with keys of its own
        _attention(name="attention_train_fp32", kind="attention_train", lens="513,1200,300", heads=8, kv_heads=8, dim=80, dtype="fp32"),
    ]


def _lens(case):
    return [int(n) for n in case["lens"].split(",")]


def _pairs(case):
    return sum(n * (n + 1) // 2 for n in _lens(case))


def _largest():
    most = {}
    for c in listed():
        k = c["kind"].split("_")[0]
        w = work(c)
        most[k] = max(most.get(k, 0), w["flops"] if k == "attention" else w["bytes"])
    return most


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = _largest()
    while True:
        kind = rng.choice(("norm", "norm_grad", "dropout", "attention", "attention", "attention_train", "attention_train"))
        if not kind.startswith("attention"):
            case = {"kind": kind, "rows": log_int(1, 16384), "cols": log_int(16, 8192)}
            if rng.random() < 0.5:
                case["cols"] = max(64, case["cols"] // 64 * 64)
            drop = rng.randint(1, 32768) / 65536
            if kind == "dropout":
                case.update(x=rng.choice(("bf16", "bf16", "fp32")), drop=drop)
            else:
                x = rng.choice(("bf16", "bf16", "fp32"))
                y = rng.choice((x, x, "e4m3")) if kind == "norm" else x
                case = _norm(**case, x=x, h=rng.choice((x, "fp32")), y=y, w=rng.choice((x, "fp32")),
                             group=rng.choice((0, 128)) if y == "e4m3" else 0, drop=rng.choice((0.0, drop)))
            if work(case)["bytes"] <= most[kind.split("_")[0]]:
                return case
            continue
        total, count = log_int(1, 16384), log_int(1, 24)
        cuts = sorted(rng.randint(0, total) for _ in range(count - 1))
        lens = [b - a for a, b in zip([0] + cuts, cuts + [total])]
        kv_heads = rng.choice((1, 2, 4, 8))
        case = _attention(kind=kind, lens=",".join(map(str, lens)), tail=rng.choice((0, 0, rng.randint(1, 100))),
                          heads=kv_heads * rng.choice((1, 2, 4, 8)), kv_heads=kv_heads, dim=rng.choice((64, 64, 128, 128, 32, 80, 96, 40)),
                          dtype=rng.choice(("bf16", "bf16", "bf16", "fp32")))
        if max(lens) <= 8192 and case["heads"] <= 32 and work(case)["flops"] <= most["attention"]:
            return case


def work(case):
    if case["kind"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * n * BYTES[case["x"]], "flops": n}
    if case["kind"].startswith("norm"):
        n, x, h, y = case["rows"] * case["cols"], BYTES[case["x"]], BYTES[case["h"]], BYTES[case["y"]]
        if case["kind"] == "norm":         # reads x, the residual, the weight; writes the sum, the output, the scales
            scales = case["rows"] * (-(-case["cols"] // case["group"]) if case["group"] else 1) * 4 if case["y"] == "e4m3" else 0
            return {"bytes": n * (x + 2 * h + y) + case["cols"] * BYTES[case["w"]] + scales, "flops": 6 * n}
        # reads the sum, both incoming gradients, the weight; writes the gradients of x, of the residual, of the weight
        return {"bytes": n * (h + y + h + x + h) + 2 * case["cols"] * BYTES[case["w"]], "flops": 12 * n}
    tokens = sum(_lens(case))
    q, kv = tokens * case["heads"] * case["dim"], tokens * case["kv_heads"] * case["dim"]
    train = case["kind"] == "attention_train"
    # forward: two products over the visible pairs; backward: five.  q, k, v, o, and their gradients once each
    return {"bytes": (2 * q + 2 * kv) * BYTES[case["dtype"]] * (2 if train else 1) + (4 * tokens * case["heads"] if train else 0),
            "flops": (14 if train else 4) * _pairs(case) * case["heads"] * case["dim"]}


# ---- inputs -------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 1000003 + 17)

    def normal(*shape, dtype, std=1.0):
        return (std * torch.randn(*shape, generator=g, device=DEV)).to(TYPES[dtype])

    def empty(*shape, dtype):
        return torch.zeros(*shape, dtype=TYPES[dtype], device=DEV)

    st = {"case": case, "seed": seed * 7919 + 3, "offset": seed % 1000}
    if case["kind"] == "dropout":
        m, n = case["rows"], case["cols"]
        return {**st, "X": normal(m, n, dtype=case["x"]), "Y": empty(m, n, dtype=case["x"])}
    if case["kind"].startswith("norm"):
        m, n = case["rows"], case["cols"]
        st["W"] = (1.0 + 0.1 * torch.randn(n, generator=g, device=DEV)).to(TYPES[case["w"]])
        if case["kind"] == "norm":
            groups = -(-n // case["group"]) if case["group"] else 1
            return {**st, "X": normal(m, n, dtype=case["x"]), "R": normal(m, n, dtype=case["h"], std=2.0), "H": empty(m, n, dtype=case["h"]),
                    "Y": empty(m, n, dtype=case["y"]), "S": empty(m, groups, dtype="fp32") if case["y"] == "e4m3" else None}
        return {**st, "H": normal(m, n, dtype=case["h"], std=2.0), "dY": normal(m, n, dtype=case["y"], std=1e-2),
                "dH": normal(m, n, dtype=case["h"], std=1e-2), "dX": empty(m, n, dtype=case["x"]), "dR": empty(m, n, dtype=case["h"]),
                "dW": empty(n, dtype=case["w"])}
    lens, t = _lens(case), case["dtype"]
    total, hq, hk, d = sum(lens) + case["tail"], case["heads"], case["kv_heads"], case["dim"]
    # query, key and value of a token stand side by side, as one projection leaves them
    qkv = normal(total, hq + 2 * hk, d, dtype=t)
    st.update(lens=lens, cu=torch.tensor([0] + lens, device=DEV).cumsum(0).to(torch.int32), Q=qkv[:, :hq], K=qkv[:, hq:hq + hk],
              V=qkv[:, hq + hk:], O=empty(total, hq, d, dtype=t), lse=empty(hq, total, dtype="fp32"))
    if case["kind"] == "attention_train":
        st.update(dO=normal(total, hq, d, dtype=t, std=1e-2), dQ=empty(total, hq, d, dtype=t), dK=empty(total, hk, d, dtype=t),
                  dV=empty(total, hk, d, dtype=t))
    return st


# ---- one pass -----------------------------------------------------------------------------------
def run(st):
    kind = st["case"]["kind"]
    return _OWN[kind](st) if own else _PLAIN[kind](st)


def _own_dropout(st):
    import paper_2605_16184_amd as ast
    ast.dropout(st["X"], st["Y"], st["case"]["drop"], seed=st["seed"], offset=st["offset"])
    return st["Y"]


def _own_norm(st):
    import paper_2605_16184_amd as ast
    c = st["case"]
    ast.rms_norm(st["X"], st["Y"], W=st["W"], R=st["R"], H=st["H"], scale=st["S"], group=c["group"], eps=EPS, p=c["drop"], seed=st["seed"],
                 offset=st["offset"])
    return [st["H"], st["Y"], st["S"]]


def _own_norm_grad(st):
    import paper_2605_16184_amd as ast
    ast.rms_norm_backward(st["H"], st["dY"], W=st["W"], dH=st["dH"], dX=st["dX"], dR=st["dR"], dW=st["dW"], eps=EPS, p=st["case"]["drop"],
                          seed=st["seed"], offset=st["offset"])
    return [st["dX"], st["dR"], st["dW"]]


def _own_attention(st):
    import paper_2605_16184_amd as ast
    ast.attention(st["Q"], st["K"], st["V"], st["O"], cu=st["cu"])
    return st["O"]


def _own_attention_train(st):
    import paper_2605_16184_amd as ast
    ast.attention(st["Q"], st["K"], st["V"], st["O"], lse=st["lse"], cu=st["cu"])
    ast.attention_backward(st["Q"], st["K"], st["V"], st["O"], st["lse"], st["dO"], st["dQ"], st["dK"], st["dV"], cu=st["cu"])
    return [st["O"], st["lse"], st["dQ"], st["dK"], st["dV"]]


# ---- plain forms --------------------------------------------------------------------------------
def _kept(st, rows, cols):
    """Which elements dropout keeps.  Element (r, c) takes 16 bits of a block of the generator Philox 4x32 with 10 rounds (Salmon,
    Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): key = seed, counter = (c // 8, r, offset), word
    (c % 8) // 2, low half first; it is kept where these are at least 65536 times the probability."""
    blocks = (cols + 7) // 8
    low = 0xFFFFFFFF
    c0 = torch.arange(blocks, device=DEV)[None, :].expand(rows, blocks)
    c1 = torch.arange(rows, device=DEV)[:, None].expand(rows, blocks)
    c2, c3 = torch.full_like(c0, st["offset"] & low), torch.full_like(c0, st["offset"] >> 32)
    k0, k1 = st["seed"] & low, st["seed"] >> 32
    for _ in range(10):
        p, q = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((q >> 32) & low) ^ c1 ^ k0, q & low, ((p >> 32) & low) ^ c3 ^ k1, p & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], dim=-1)
    bits = torch.stack([words & 0xFFFF, words >> 16], dim=-1).reshape(rows, blocks * 8)[:, :cols]
    return bits >= round(st["case"]["drop"] * 65536)


def _dropped(st, x):
    if st["case"]["drop"] == 0:
        return x
    return torch.where(_kept(st, *x.shape), x * (1.0 / (1.0 - st["case"]["drop"])), 0.0)


def _plain_dropout(st):
    return _dropped(st, st["X"].float()).to(st["X"].dtype)


def _plain_norm(st):
    c = st["case"]
    h = st["R"].float() + _dropped(st, st["X"].float())
    y = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS) * st["W"].float()
    if c["y"] != "e4m3":
        return [h.to(st["H"].dtype), y.to(st["Y"].dtype), None]
    rows, cols = y.shape
    group = c["group"] or cols
    groups = -(-cols // group)
    z = torch.zeros(rows, groups * group, device=y.device)
    z[:, :cols] = y
    z = z.view(rows, groups, group)
    scale = z.abs().amax(dim=2).clamp_min(SCALE_FLOOR) / E4M3_MAX
    q = (z / scale[:, :, None]).view(rows, groups * group)[:, :cols]
    return [h.to(st["H"].dtype), q.contiguous().to(torch.float8_e4m3fn), scale]


def _plain_norm_grad(st):
    h, dy, w = st["H"].float(), st["dY"].float(), st["W"].float()
    r = torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS)
    dn = dy * w
    dr = st["dH"].float() + r * (dn - h * (r * r) * (dn * h).mean(dim=1, keepdim=True))
    dw = (dy * h * r).sum(dim=0)
    return [_dropped(st, dr).to(st["dX"].dtype), dr.to(st["dR"].dtype), dw.to(st["dW"].dtype)]


def _plain_attention(st, train=False):
    c = st["case"]
    hq, hk, d = c["heads"], c["kv_heads"], c["dim"]
    g, scale = hq // hk, 1.0 / math.sqrt(d)
    out = {k: torch.zeros_like(st[k]) for k in ("O", "lse", "dQ", "dK", "dV") if k in st}
    at = 0
    for n in st["lens"]:
        s = slice(at, at + n)
        at += n
        if n == 0:
            continue
        # kv_heads x (heads of the group x tokens) x dim
        q = st["Q"][s].float().permute(1, 0, 2).reshape(hk, g * n, d)
        k, v = st["K"][s].float().permute(1, 0, 2).contiguous(), st["V"][s].float().permute(1, 0, 2).contiguous()
        later = torch.arange(n, device=q.device)[None, :] > torch.arange(n, device=q.device)[:, None]
        z = (q @ k.transpose(1, 2).contiguous() * scale).view(hk, g, n, n).masked_fill_(later, -math.inf)
        m = z.amax(dim=-1, keepdim=True)
        p = torch.exp(z - m)
        del z
        total = p.sum(dim=-1, keepdim=True)
        p = (p / total).view(hk, g * n, n)
        o = p @ v
        out["O"][s] = o.view(hq, n, d).permute(1, 0, 2).to(out["O"].dtype)
        if not train:
            continue
        out["lse"][:, s] = (m + torch.log(total)).view(hq, n)
        do = st["dO"][s].float().permute(1, 0, 2).reshape(hk, g * n, d)
        ds = do @ v.transpose(1, 2).contiguous() - (do * o).sum(dim=-1, keepdim=True)
        ds = ds * p * scale
        out["dQ"][s] = (ds @ k).view(hq, n, d).permute(1, 0, 2).to(out["dQ"].dtype)
        out["dK"][s] = (ds.transpose(1, 2).contiguous() @ q).permute(1, 0, 2).to(out["dK"].dtype)
        out["dV"][s] = (p.transpose(1, 2).contiguous() @ do).permute(1, 0, 2).to(out["dV"].dtype)
    return [out[k] for k in ("O", "lse", "dQ", "dK", "dV")] if train else out["O"]


def _plain_attention_train(st):
    return _plain_attention(st, train=True)


_OWN = {"dropout": _own_dropout, "norm": _own_norm, "norm_grad": _own_norm_grad, "attention": _own_attention,
        "attention_train": _own_attention_train}
_PLAIN = {"dropout": _plain_dropout, "norm": _plain_norm, "norm_grad": _plain_norm_grad, "attention": _plain_attention,
          "attention_train": _plain_attention_train}


# ---- in 64 bits ---------------------------------------------------------------------------------
def _mask64(seed, offset, rows, cols, drop):
    """The factors of dropout in 64 bits: 0 or 1 / (1 - drop), with the generator's state as four numbers for every eight columns."""
    mask32 = (1 << 32) - 1
    row = torch.arange(rows, device=DEV).view(-1, 1)
    col = torch.arange(0, cols, 8, device=DEV).view(1, -1) // 8
    zero = torch.zeros(rows, col.shape[1], dtype=torch.int64, device=DEV)
    state = [zero + col, zero + row, zero + (offset & mask32), zero + (offset >> 32)]
    key = [seed & mask32, seed >> 32]

    def wide(a, x):                        # high and low word of a 32 x 32 bit product, by halves: nothing passes 63 bits
        lo, hi = a * (x & 0xFFFF), a * (x >> 16)
        t = hi + (lo >> 16)
        return t >> 16, ((t & 0xFFFF) << 16) | (lo & 0xFFFF)

    for i in range(10):
        h0, l0 = wide(0xD2511F53, state[0])
        h2, l2 = wide(0xCD9E8D57, state[2])
        state = [h2 ^ state[1] ^ key[0], l2, h0 ^ state[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) & mask32, (key[1] + 0xBB67AE85) & mask32]
    u = torch.empty(rows, col.shape[1], 8, dtype=torch.int64, device=DEV)
    for i in range(8):
        u[:, :, i] = (state[i // 2] >> (16 * (i % 2))) & 0xFFFF
    keep = u.view(rows, -1)[:, :cols] >= int(drop * 65536 + 0.5)
    return keep.double() / (1.0 - drop)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"].startswith("attention"):
        return _exact_attention(case, st)
    factor = _mask64(st["seed"], st["offset"], case["rows"], case["cols"], case["drop"]) if case["drop"] else 1.0
    if case["kind"] == "dropout":
        return st["X"].double() * factor
    w = st["W"].double()
    if case["kind"] == "norm":
        h = st["X"].double() * factor + st["R"].double()
        y = w * h / torch.sqrt(h.square().sum(1, keepdim=True) / case["cols"] + EPS)
        if case["y"] != "e4m3":
            return [h, y, None]
        scales, parts = [], []
        for part in y.split(case["group"] or case["cols"], dim=1):
            scales.append(torch.clamp(part.abs().max(dim=1).values, min=SCALE_FLOOR) / E4M3_MAX)
            parts.append(part / scales[-1].view(-1, 1))
        return [h, torch.cat(parts, 1), torch.stack(scales, 1)]
    # y = w n, n = h / s, s = sqrt(mean h^2 + eps):  dn = w dy,  dh = (dn - n <dn, n> / cols) / s
    h = st["H"].double()
    s = torch.sqrt(h.square().sum(1, keepdim=True) / case["cols"] + EPS)
    n, dn = h / s, st["dY"].double() * w
    dh = st["dH"].double() + (dn - n * (dn * n).sum(1, keepdim=True) / case["cols"]) / s
    return [dh * factor, dh, (st["dY"].double() * n).sum(0)]


def _exact_attention(case, st):
    train = case["kind"] == "attention_train"
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    res = {k: torch.zeros(st[k].shape, dtype=torch.float64, device=DEV) for k in ("O", "lse", "dQ", "dK", "dV") if k in st}
    start = 0
    for n in st["lens"]:
        end = start + n
        for j in range(hq if n else 0):
            kv = j * hk // hq
            q, k, v = st["Q"][start:end, j].double(), st["K"][start:end, kv].double(), st["V"][start:end, kv].double()
            z = torch.mm(q, k.t().contiguous()) / math.sqrt(d)
            z = z + torch.full((n, n), -math.inf, dtype=torch.float64, device=DEV).triu(1)
            lse = torch.logsumexp(z, dim=1)
            p = torch.exp(z - lse[:, None])
            res["O"][start:end, j] = torch.mm(p, v)
            if train:
                do = st["dO"][start:end, j].double()
                dp = torch.mm(do, v.t().contiguous())
                dz = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
                res["lse"][j, start:end] = lse
                res["dQ"][start:end, j] = torch.mm(dz, k)
                res["dK"][start:end, kv] += torch.mm(dz.t().contiguous(), q)
                res["dV"][start:end, kv] += torch.mm(p.t().contiguous(), do)
        start = end
    return [res[k] for k in ("O", "lse", "dQ", "dK", "dV")] if train else res["O"]
