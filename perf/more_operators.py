"""The operators of a layer of experts as measured cases: routing, quantize, scaled_matmul and combine.

`routing` scores the experts of every token, picks some of them and plans their rows expert by expert; `quantize` turns
rows (or gated pairs of rows, or weights) into 8-bit codes with a scale for each block of 128 and spreads them to the
experts' rows; `scaled_matmul` is the product of such codes, one weight or one per group of rows; `combine` adds up every
token's results by weight.  `run` computes one of them, in elementary torch operations (`own = False`) or through the library.
"""
import math
import random

import numpy as np
import torch

own = False

F32, BF16, F64, I32, E4M3 = torch.float32, torch.bfloat16, torch.float64, torch.int32, torch.float8_e4m3fn
BLOCK = 128


# ------------------------------------------------------------------------------------------------- the cases

def _routing(name, tokens, experts, top_k, scoring, biased, groups, top_groups, renormalise, dtype, pad):
    return {"name": name, "op": "routing", "tokens": tokens, "experts": experts, "top_k": top_k, "scoring": scoring, "biased": biased,
            "groups": groups, "top_groups": top_groups, "renormalise": renormalise, "dtype": dtype, "pad": pad}


def _quantize(name, rows, cols, dtype, gated, copies, block_rows):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "gated": gated, "copies": copies, "block_rows": block_rows}


def _scaled(name, rows, groups, n, k, dtype):
    return {"name": name, "op": "scaled_matmul", "rows": rows, "groups": groups, "n": n, "k": k, "dtype": dtype}


def _combine(name, tokens, top_k, cols, dtype, based, pad):
    return {"name": name, "op": "combine", "tokens": tokens, "top_k": top_k, "cols": cols, "dtype": dtype, "based": based, "pad": pad}


def listed():
    return [
        # one token of a decoding step: the smallest call
        _routing("route 1 token", 1, 64, 6, "softmax", False, 1, 1, False, "bf16", 0),
        # a decoding batch padded to a fixed size, balanced by a bias, experts in groups
        _routing("route 64 tokens", 61, 256, 8, "sigmoid", True, 8, 4, True, "f32", 3),
        # a full prompt batch with the same router, an odd number of tokens
        _routing("route 8191 tokens", 8191, 256, 8, "sigmoid", True, 8, 4, True, "f32", 1),
        # the activations of a prompt batch, sent to eight experts each
        _quantize("quantize 8192 tokens to 8 rows each", 8192, 4096, "bf16", False, 8, 1),
        # between an expert's two products: gate and up columns, an odd number of rows
        _quantize("gate and quantize 49157 rows", 49157, 1408, "bf16", True, 0, 1),
        # weights when a model is loaded
        _quantize("quantize weights 11008 x 4096", 11008, 4096, "f32", False, 0, 128),
        # one token through one dense layer: latency and the weights' bytes
        _scaled("1 row, 4096 to 11008", 1, 1, 11008, 4096, "bf16"),
        # a decoding batch of 64 tokens with 8 experts each: every expert's weights for a few rows
        _scaled("512 rows of 128 experts, 4096 to 2816", 512, 128, 2816, 4096, "bf16"),
        # a prompt batch of 8192 tokens with 8 experts each, as uneven as a router leaves it
        _scaled("65536 rows of 64 experts, 4096 to 2816", 65536, 64, 2816, 4096, "bf16"),
        # a prompt batch through one dense layer
        _scaled("8192 rows, 4096 to 11008", 8192, 1, 11008, 4096, "bf16"),
        # the end of a decoding step's layer
        _combine("combine 64 tokens of 6", 64, 6, 4096, "bf16", False, 0),
        # the end of a prompt batch's layer, added to the residual stream
        _combine("combine 8192 tokens of 8", 8192, 8, 4096, "bf16", True, 0),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("routing", "quantize", "scaled_matmul", "scaled_matmul", "combine"))
    if op == "routing":
        experts = rng.choice((8, 16, 60, 64, 128, 160, 256, 256))
        groups = rng.choice((1, 4)) if experts < 64 else rng.choice((1, 4, 8))
        groups = groups if experts % groups == 0 else 1
        top_groups = rng.randint(max(1, groups // 2), groups)
        top_k = rng.randint(1, min(8, top_groups * (experts // groups)))
        c = _routing("", _log(rng, 1, 8192), experts, top_k, rng.choice(("softmax", "sigmoid")), rng.random() < 0.6, groups, top_groups,
                     rng.random() < 0.7, rng.choice(("bf16", "f32")), rng.choice((0, rng.randint(1, 40))))
    elif op == "quantize":
        while True:
            cols = 16 * _log(rng, 8, 512)
            kind = rng.choice(("spread", "spread", "gated", "weights"))
            rows = _log(rng, 1, 11008 if kind == "weights" else 8192 if kind == "spread" else 49157)
            copies = rng.randint(0, 8) if kind == "spread" else 0
            if rows * cols * max(1, copies) <= 65536 * 4096:
                break
        c = _quantize("", rows, cols, rng.choice(("bf16", "bf16", "f32")), kind == "gated", copies, 128 if kind == "weights" else 1)
    elif op == "scaled_matmul":
        while True:
            groups = rng.choice((1, 1, 8, 32, 60, 64, 128))
            rows = _log(rng, 1, 65536)
            n, k = rng.choice((640, 1408, 2048, 2816, 4096, 11008, 8 * _log(rng, 16, 512))), rng.choice((512, 1408, 2048, 4096, 4096, 16 * _log(rng, 8, 256)))
            # no more products, and no more weights, than the largest listed cases
            if rows * n * k <= 65536 * 2816 * 4096 and groups * n * k <= 128 * 2816 * 4096:
                break
        c = _scaled("", rows, groups, n, k, rng.choice(("bf16", "bf16", "f32")))
    else:
        c = _combine("", _log(rng, 1, 8192), rng.randint(1, 8), 8 * _log(rng, 16, 512), rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.5,
                     rng.choice((0, rng.randint(1, 40))))
    del c["name"]
    return c


def _up(a, b):
    return -(-a // b)


def _counts(case):
    """Rows of every group: a function of the case alone, as uneven as a router without a balancing bias leaves them."""
    rows, groups = case["rows"], case["groups"]
    r = np.random.default_rng([rows, groups, case["n"]])
    p = np.exp(0.5 * r.standard_normal(groups))
    return r.multinomial(rows, p / p.sum()) if groups > 1 else np.array([rows])


# ------------------------------------------------------------------------------------------------- the inputs

def _normal(g, shape, dtype=F32, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=F32, device="cuda").normal_(mean, std, generator=g).to(dtype)


def _dtype(case):
    return BF16 if case["dtype"] == "bf16" else F32


def _codes(g, rows, cols, block_rows, std):
    """Normal values as 8-bit codes with their scales: [rows, cols], [rows / block_rows, cols / 128]."""
    kb, rb = _up(cols, BLOCK), _up(rows, block_rows)
    x = torch.zeros((rb * block_rows, kb * BLOCK), dtype=F32, device="cuda")
    x[:rows, :cols].normal_(0, std, generator=g)
    x = x.view(rb, block_rows, kb, BLOCK)
    s = x.abs().amax((1, 3)).div_(448.0).clamp_(min=2.0 ** -126)
    return x.div_(s[:, None, :, None]).to(E4M3).view(rb * block_rows, kb * BLOCK)[:rows, :cols].contiguous(), s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = dict(case)
    if own:
        import paper_2603_24239_b200 as dvm
    if case["op"] == "routing":
        t, e, k = case["tokens"] + case["pad"], case["experts"], case["top_k"]
        positions = torch.arange(t, dtype=I32, device="cuda")
        positions[case["tokens"]:] = -1   # rows behind the last token of a padded batch
        s.update(rows=t, logits=_normal(g, (t, e), _dtype(case), 1.5), bias=_normal(g, (e,), F32, 0.05), positions=positions, factor=2.5 if case["renormalise"] else 1.0,
                 ids=torch.empty((t, k), dtype=I32, device="cuda"), weights=torch.empty((t, k), device="cuda"),
                 places=torch.empty((t, k), dtype=I32, device="cuda"), starts=torch.empty(e + 1, dtype=I32, device="cuda"))
        if own:
            s["code"] = dvm.encode_routing(s["logits"], k, scoring=case["scoring"], biased=case["biased"], groups=case["groups"], top_groups=case["top_groups"],
                                           renormalise=case["renormalise"], factor=s["factor"], masked=True)
            s["workspace"] = torch.empty(max(16, dvm.tensor_extents(s["code"])[-1]), dtype=torch.uint8, device="cuda")
    elif case["op"] == "quantize":
        rows, cols, copies, br = case["rows"], case["cols"], case["copies"], case["block_rows"]
        x = _normal(g, (rows, cols * (2 if case["gated"] else 1)), F32, 1.0 if br == 1 else 0.02)
        if br == 1:   # some channels of activations are far larger than the others
            x *= torch.exp(_normal(g, (x.shape[1],), F32, 0.5))
        out_rows = rows * max(1, copies)
        s.update(x=x.to(_dtype(case)), codes=torch.zeros((out_rows, cols), dtype=E4M3, device="cuda"),
                 scales=torch.zeros((_up(out_rows, br), _up(cols, BLOCK)), device="cuda"),
                 places=torch.randperm(out_rows, generator=g, device="cuda").to(I32).view(rows, copies) if copies else None)
        if own:
            s["code"] = dvm.encode_quantize(s["x"], s["codes"], s["scales"], places=s["places"], gated=case["gated"], block_rows=br)
    elif case["op"] == "scaled_matmul":
        rows, groups, n, k = case["rows"], case["groups"], case["n"], case["k"]
        x, xs = _codes(g, rows, k, 1, 1.0)
        w = torch.empty((groups, n, k), dtype=E4M3, device="cuda")
        ws = torch.empty((groups, _up(n, BLOCK), _up(k, BLOCK)), device="cuda")
        for i in range(groups):
            w[i], ws[i] = _codes(g, n, k, BLOCK, 1.0 / math.sqrt(k))
        counts = _counts(case)
        starts = np.concatenate([[0], np.cumsum(counts)])
        s.update(x=x, xs=xs, w=w, ws=ws, starts=torch.tensor(starts, dtype=I32, device="cuda"), most=int(counts.max()),
                 out=torch.zeros((rows, n), dtype=_dtype(case), device="cuda"))
        if own:
            s["code"] = dvm.encode_scaled_matmul(x, xs, w, ws, s["out"], starts=s["starts"] if groups > 1 else None)
            s["workspace"] = torch.empty(max(16, dvm.tensor_extents(s["code"])[-1]), dtype=torch.uint8, device="cuda")
    else:
        t, k, cols = case["tokens"] + case["pad"], case["top_k"], case["cols"]
        rows = case["tokens"] * k
        places = torch.full((t, k), -1, dtype=I32, device="cuda")
        places[:case["tokens"]] = torch.randperm(rows, generator=g, device="cuda").to(I32).view(-1, k)
        weights = torch.rand((t, k), generator=g, device="cuda") + 0.05
        s.update(y=_normal(g, (rows, cols), _dtype(case)), places=places, weights=weights / weights.sum(1, keepdim=True),
                 base=_normal(g, (t, cols), _dtype(case)), out=torch.zeros((t, cols), dtype=_dtype(case), device="cuda"))
        if own:
            s["code"] = dvm.encode_combine(s["y"], s["places"], s["weights"], s["out"], base=s["base"] if case["based"] else None)
    return s


# ------------------------------------------------------------------------------------------------- one pass

def run(s):
    return {"routing": _run_routing, "quantize": _run_quantize, "scaled_matmul": _run_scaled, "combine": _run_combine}[s["op"]](s)


def _run_routing(s):
    if own:
        import paper_2603_24239_b200 as dvm
        bias = (s["bias"],) if s["biased"] else ()
        dvm.launch(s["code"], (s["logits"], *bias, s["positions"], s["ids"], s["weights"], s["places"], s["starts"], s["workspace"]))
        return {k: s[k] for k in ("ids", "weights", "places", "starts")}
    t, e, k, groups = s["rows"], s["experts"], s["top_k"], s["groups"]
    x = s["logits"].double()   # 64 bits: two experts may be nearer than 32 bits tell apart
    if s["scoring"] == "softmax":
        p = (x - x.amax(1, keepdim=True)).exp()
        score = p / p.sum(1, keepdim=True)
    else:
        score = 1.0 / (1.0 + (-x).exp())
    choice = score + s["bias"].double() if s["biased"] else score
    if groups > 1:
        of = choice.view(t, groups, e // groups).sort(2, descending=True)[0][..., :2].sum(2)
        best = of.sort(dim=1, descending=True, stable=True)[1][:, :s["top_groups"]]
        allowed = torch.zeros((t, groups), dtype=torch.bool, device=x.device).scatter_(1, best, True)
        choice = torch.where(allowed.repeat_interleave(e // groups, 1), choice, -math.inf)
    ids = choice.sort(dim=1, descending=True, stable=True)[1][:, :k]
    weights = score.gather(1, ids).float()
    if s["renormalise"]:
        weights = weights / weights.sum(1, keepdim=True)
    real = (s["positions"] >= 0)[:, None]
    ids = torch.where(real, ids, e)
    by_expert, order = ids.reshape(-1).sort(stable=True)
    places = torch.empty_like(order)
    places[order] = torch.arange(t * k, device=x.device)
    starts = torch.searchsorted(by_expert, torch.arange(e + 1, device=x.device))
    return {"ids": torch.where(real, ids, -1).to(I32), "weights": torch.where(real, weights * s["factor"], 0.0),
            "places": torch.where(real, places.view(t, k), -1).to(I32), "starts": starts.to(I32)}


def _nearest_code(v):
    """The e4m3 value nearest to v (64 bits; ties to even), as a tensor of codes: steps of 2^-3 of the value's power of two, 2^-9 at least."""
    step = torch.exp2(torch.frexp(v)[1].clamp(min=-5).double() - 4)
    return (torch.round(v / step) * step).clamp(-448.0, 448.0).to(E4M3)


def _run_quantize(s):
    if own:
        import paper_2603_24239_b200 as dvm
        places = () if s["places"] is None else (s["places"],)
        dvm.launch(s["code"], (s["x"], *places, s["codes"], s["scales"]))
        return {"codes": s["codes"], "scales": s["scales"]}
    rows, cols, br = s["rows"], s["cols"], s["block_rows"]
    x = s["x"].float()
    if s["gated"]:
        x = x[:, :cols] / (1.0 + (-x[:, :cols]).exp()) * x[:, cols:]
    kb, rb = _up(cols, BLOCK), _up(rows, br)
    v = torch.zeros((rb * br, kb * BLOCK), dtype=F32, device=x.device)
    v[:rows, :cols] = x
    v = v.view(rb, br, kb, BLOCK)
    scales = (v.abs().amax((1, 3)).double() / 448.0).float().clamp(min=2.0 ** -126)   # (64 bits: quotients often lie on a border between two codes)
    codes = _nearest_code(v.double() / scales.double()[:, None, :, None]).view(rb * br, kb * BLOCK)[:rows, :cols]
    if s["places"] is None:
        return {"codes": codes.contiguous(), "scales": scales}
    for_row = torch.empty(rows * s["copies"], dtype=torch.int64, device=x.device)
    for_row[s["places"].reshape(-1).long()] = torch.arange(rows, device=x.device).repeat_interleave(s["copies"])
    return {"codes": codes.view(torch.uint8)[for_row].view(E4M3), "scales": scales[for_row]}


def _run_scaled(s):
    if own:
        import paper_2603_24239_b200 as dvm
        starts = (s["starts"],) if s["groups"] > 1 else ()
        dvm.launch(s["code"], (s["x"], s["xs"], s["w"], s["ws"], *starts, s["out"], s["workspace"]))
        return s["out"]
    rows, groups, n, k = s["rows"], s["groups"], s["n"], s["k"]
    x = s["x"].float() * s["xs"].repeat_interleave(BLOCK, 1)[:, :k]
    w = s["w"].float()
    w *= s["ws"].repeat_interleave(BLOCK, 1)[:, :n].repeat_interleave(BLOCK, 2)[:, :, :k]
    if groups == 1:
        return torch.matmul(x, w[0].t()).to(s["out"].dtype)
    # the rows of every group behind one another, padded to the longest
    first = s["starts"][:-1].long()
    at = (first[:, None] + torch.arange(s["most"], device=x.device)[None, :]).clamp(max=rows - 1)
    y = torch.matmul(x[at], w.transpose(1, 2))
    r = torch.arange(rows, device=x.device)
    group = torch.searchsorted(s["starts"][1:].long().contiguous(), r, right=True)
    return y[group, r - first[group]].to(s["out"].dtype)


def _run_combine(s):
    if own:
        import paper_2603_24239_b200 as dvm
        base = (s["base"],) if s["based"] else ()
        dvm.launch(s["code"], (s["y"], s["places"], s["weights"], *base, s["out"]))
        return s["out"]
    t = s["tokens"]   # the rows behind them are padding and stay as they are
    v = (s["y"].float()[s["places"][:t].long()] * s["weights"][:t, :, None]).sum(1)
    if s["based"]:
        v = v + s["base"][:t].float()
    s["out"][:t] = v.to(s["out"].dtype)
    return s["out"]


# ------------------------------------------------------------------------------------------------- exact values, work

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "routing":
        t, e, k, per = case["tokens"], case["experts"], case["top_k"], case["experts"] // case["groups"]
        z = s["logits"][:t].to(F64)
        score = torch.softmax(z, 1) if case["scoring"] == "softmax" else torch.sigmoid(z)
        pick = (score + s["bias"].to(F64) if case["biased"] else score).clone()
        if per < e:
            strength = pick.view(t, -1, per).topk(min(2, per), 2).values.sum(2)
            least = strength.topk(case["top_groups"], 1).values[:, -1:]
            pick.view(t, -1, per)[strength < least] = -math.inf
        chosen = []
        for _ in range(k):
            best = pick.max(1, keepdim=True).indices
            chosen.append(score.gather(1, best))
            pick.scatter_(1, best, -math.inf)
        w = torch.cat(chosen, 1)
        w = (w / w.sum(1, keepdim=True) if case["renormalise"] else w) * s["factor"]
        return {"ids": None, "weights": torch.cat([w, w.new_zeros((case["pad"], k))]), "places": None, "starts": None}
    if case["op"] == "quantize":
        rows, cols, br = case["rows"], case["cols"], case["block_rows"]
        v = s["x"].to(F64)
        if case["gated"]:
            v = torch.sigmoid(v[:, :cols]) * v[:, :cols] * v[:, cols:]
        v = torch.nn.functional.pad(v, (0, -cols % BLOCK, 0, -rows % br))
        a = v.abs().view(v.shape[0] // br, br, -1, BLOCK).amax(3).amax(1)
        scales = (a / 448.0).clamp(min=2.0 ** -126)
        # the codes' values lie in a table; each quotient goes to the nearest
        table = torch.arange(127, dtype=torch.uint8, device="cuda").view(E4M3).to(F64)
        codes = torch.empty((rows, cols), dtype=F64, device="cuda")
        wide = scales.to(F32).to(F64).repeat_interleave(br, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]
        for b in range(0, rows, 4096):
            x = v[b: min(rows, b + 4096), :cols] / wide[b: b + 4096]
            m = x.abs().clamp(max=448.0)
            hi = torch.searchsorted(table, m).clamp(1, 126)
            lo = hi - 1
            up = m - table[lo] - (table[hi] - m)
            at = torch.where((up > 0) | ((up == 0) & (hi % 2 == 0)), hi, lo)
            codes[b: b + 4096] = torch.where(x < 0, -table[at], table[at])
        if case["copies"]:
            p = s["places"].long()
            full, fs = torch.empty((rows * case["copies"], cols), dtype=F32, device="cuda"), torch.empty((rows * case["copies"], scales.shape[1]), dtype=F64, device="cuda")
            for j in range(case["copies"]):
                full[p[:, j]], fs[p[:, j]] = codes.to(F32), scales
            codes, scales = full.to(F64), fs
        return {"codes": codes, "scales": scales}
    if case["op"] == "scaled_matmul":
        n, k = case["n"], case["k"]
        out = torch.empty((case["rows"], n), dtype=F64, device="cuda")
        col = torch.arange(k, device="cuda") // BLOCK
        row = torch.arange(n, device="cuda") // BLOCK
        a = 0
        for g, count in enumerate(_counts(case).tolist()):
            if count:
                w = s["w"][g].to(F64) * s["ws"][g].to(F64)[row[:, None], col[None, :]]
                for b in range(a, a + count, 8192):
                    c = min(a + count, b + 8192)
                    out[b:c] = (s["x"][b:c].to(F64) * s["xs"][b:c].to(F64)[:, col]) @ w.T
            a += count
        return out
    t = case["tokens"]
    out = s["out"].to(F64)
    acc = s["base"][:t].to(F64) if case["based"] else torch.zeros_like(out[:t])
    for j in range(case["top_k"]):
        acc = acc + s["weights"][:t, j, None].to(F64) * s["y"][s["places"][:t, j].long()].to(F64)
    out[:t] = acc
    return out


def work(case):
    es = 2 if case.get("dtype") == "bf16" else 4
    if case["op"] == "routing":
        t, all_rows, e, k = case["tokens"], case["tokens"] + case["pad"], case["experts"], case["top_k"]
        return {"bytes": t * e * es + (4 * e if case["biased"] else 0) + 4 * all_rows + 12 * all_rows * k + 4 * (e + 1), "flops": 6 * t * e}
    if case["op"] == "quantize":
        rows, cols, br = case["rows"], case["cols"], case["block_rows"]
        to = rows * max(1, case["copies"])
        return {"bytes": rows * cols * es * (2 if case["gated"] else 1) + 4 * rows * case["copies"] + to * cols + 4 * _up(to, br) * _up(cols, BLOCK),
                "flops": rows * cols * (7 if case["gated"] else 3)}
    if case["op"] == "scaled_matmul":
        rows, n, k = case["rows"], case["n"], case["k"]
        used = int((_counts(case) > 0).sum())
        return {"bytes": rows * k + 4 * rows * _up(k, BLOCK) + used * (n * k + 4 * _up(n, BLOCK) * _up(k, BLOCK)) + rows * n * es
                + (4 * (case["groups"] + 1) if case["groups"] > 1 else 0), "flops": 2 * rows * n * k}
    t, all_rows, k, cols = case["tokens"], case["tokens"] + case["pad"], case["top_k"], case["cols"]
    return {"bytes": t * (k + 1 + (1 if case["based"] else 0)) * cols * es + 8 * all_rows * k, "flops": 2 * t * k * cols}
