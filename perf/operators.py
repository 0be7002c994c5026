"""The serving operators of the library as measured cases: paging, rotary and attention.

`paging` gives every new token of a batch its row, position and cache slot and hands out cache pages; `rotary`
normalises the query and key heads, rotates them by position and writes keys and values into the paged cache;
`attention` is causal attention of the new tokens over that cache with a sliding window and first tokens that stay
visible.  `run` computes one of them, in elementary torch operations (`own = False`) or through the library.
"""
import math
import random

import numpy as np
import torch

own = False

F32, BF16 = torch.float32, torch.bfloat16


# ------------------------------------------------------------------------------------------------- the cases

def _paging(name, requests, fresh, held, page, pad):
    return {"name": name, "op": "paging", "requests": requests, "fresh": fresh, "held": held, "page": page, "pad": pad}


def _rotary(name, tokens, q_heads, kv_heads, dim, rot, norm, interleaved, dtype, page, pad):
    return {"name": name, "op": "rotary", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "rot": rot, "norm": norm, "interleaved": interleaved, "dtype": dtype, "page": page, "pad": pad}


def _attention(name, requests, fresh, held, q_heads, kv_heads, dim, page, window, sinks, heads_first):
    return {"name": name, "op": "attention", "requests": requests, "fresh": fresh, "held": held, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "page": page, "window": window, "sinks": sinks, "heads_first": heads_first}


def listed():
    return [
        # a decoding step of a small batch: one new token for every request, the smallest call
        _paging("paging 32 single tokens", 32, 1, 8192, 16, 0),
        # a step that admits many prompts of mixed lengths, rows padded to a fixed batch
        _paging("paging 256 prompts", 256, 1024, 2048, 16, 173),
        # one token of one request, multi-head layout: latency
        _rotary("rotary 1 token", 1, 32, 32, 128, 128, True, False, "bf16", 16, 0),
        # a full prompt batch with shared key heads
        _rotary("rotary 8192 tokens", 8192, 32, 8, 128, 128, True, False, "bf16", 64, 0),
        # fp32 activations, part of the head rotated, neighbouring pairs, an odd number of rows with padding behind
        _rotary("rotary 1531 tokens fp32", 1531, 40, 8, 96, 64, True, True, "f32", 16, 5),
        # one long prompt, no window: what a first request costs
        _attention("prompt 8192", 1, 8192, 0, 32, 8, 128, 64, 0, 0, True),
        # a long prompt under a sliding window with four sinks
        _attention("prompt 8192 window 1024", 1, 8192, 0, 32, 32, 128, 16, 1024, 4, False),
        # ragged prompts that continue cached prefixes, odd head size and group
        _attention("12 ragged prompts", 12, 700, 1300, 40, 8, 96, 16, 0, 0, False),
        # small heads, a window shorter than a page row of tiles
        _attention("prompts 64-wide window 128", 8, 1531, 300, 16, 4, 64, 32, 128, 1, True),
        # one request, one token: the latency of a decoding step
        _attention("1 single token", 1, 1, 8192, 32, 8, 128, 16, 0, 0, True),
        # a decoding batch of ragged lengths over the whole context
        _attention("64 single tokens", 64, 1, 8192, 64, 8, 128, 16, 0, 0, True),
        # a decoding batch of long contexts under a window with sinks, key and value heads not shared
        _attention("32 single tokens window 4096", 32, 1, 16384, 32, 32, 128, 64, 4096, 4, False),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("paging", "rotary", "attention", "attention"))
    if op == "paging":
        single = rng.random() < 0.4
        requests = _log(rng, 1, 512)
        fresh = 1 if single else _log(rng, 2, 1024)
        c = _paging("", requests, fresh, _log(rng, 1, 8192), rng.choice((16, 32, 64, 128)), rng.choice((0, rng.randint(1, 300))))
    elif op == "rotary":
        dim = rng.choice((64, 80, 96, 128, 128))
        kv = rng.choice((1, 2, 4, 8, 32))
        group = rng.randint(1, max(1, 40 // kv))
        rot = rng.choice((dim, dim, dim // 2))
        tokens = _log(rng, 1, 8192)
        c = _rotary("", tokens, kv * group, kv, dim, rot, rng.random() < 0.8, rng.random() < 0.4,
                    rng.choice(("bf16", "bf16", "f32")), rng.choice((16, 32, 64)), rng.choice((0, rng.randint(1, 50))))
    else:
        while True:
            dim = rng.choice((64, 80, 96, 128, 128))
            kv = rng.choice((1, 2, 4, 8, 8, 32))
            group = rng.randint(1, max(1, min(16, 64 // kv)))
            window = rng.choice((0, 0, _log(rng, 16, 4096)))
            sinks = rng.choice((0, rng.randint(1, 64))) if window else 0
            if rng.random() < 0.5:
                requests, fresh, held = _log(rng, 1, 96), 1, _log(rng, 1, 16384)
            else:
                requests, fresh, held = _log(rng, 1, 16), _log(rng, 2, 4096), rng.choice((0, _log(rng, 1, 4096)))
            # no more scores, and no more cache, than the largest listed cases
            if requests * fresh * (fresh + held) * kv * group <= 1 << 31 and requests * (held + fresh) * kv * dim <= 1 << 29:
                break
        c = _attention("", requests, fresh, held, kv * group, kv, dim, rng.choice((16, 32, 64, 128)), window, sinks, rng.random() < 0.5)
    del c["name"]
    return c


def _lengths(case):
    """(cached, fresh) tokens of every request: a function of the case alone.  One request has the full lengths."""
    n, fresh, held = case["requests"], case["fresh"], case["held"]
    r = random.Random("lengths %d %d %d" % (n, fresh, held))
    f = [fresh] + [fresh if fresh == 1 else r.randint(max(1, fresh // 8), fresh) for _ in range(n - 1)]
    c = [held] + [r.randint(held // 4, held) if held else 0 for _ in range(n - 1)]
    order = list(range(n))
    r.shuffle(order)
    return np.array([c[i] for i in order], dtype=np.int64), np.array([f[i] for i in order], dtype=np.int64)


def _blocks(tokens, page):
    return -(-tokens // page)


# ------------------------------------------------------------------------------------------------- the inputs

def _normal(g, shape, dtype, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=F32, device="cuda").normal_(mean, std, generator=g).to(dtype)


def _ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _angles(rows, rot):
    """cos and sin of position x base^(-2 k / rot), made in 64 bits: [rows, rot] = [cos | sin]."""
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * inv[None, :]
    return torch.cat([a.cos(), a.sin()], 1).to(F32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    host = random.Random(int(seed))
    s = dict(case)
    page = case["page"]
    if case["op"] == "paging":
        cached, fresh = _lengths(case)
        n = case["requests"]
        width = int(_blocks(cached + fresh, page).max()) + 2
        held = _blocks(cached, page)
        new = int((_blocks(cached + fresh, page) - held).sum())
        pool = torch.randperm(int(held.sum()) + new + 7, generator=g, device="cuda").to(torch.int32)
        table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        table[torch.arange(width, device="cuda")[None, :] < _ints(held)[:, None]] = pool[: int(held.sum())]
        rows = int(fresh.sum()) + case["pad"]
        s.update(cached=_ints(cached), new=_ints(fresh), free=pool[int(held.sum()):].contiguous(), table=table, rows=rows, width=width,
                 starts=torch.empty(n + 1, dtype=torch.int32, device="cuda"), lengths=torch.empty(n, dtype=torch.int32, device="cuda"),
                 positions=torch.empty(rows, dtype=torch.int32, device="cuda"), slots=torch.empty(rows, dtype=torch.int32, device="cuda"),
                 taken=torch.empty(1, dtype=torch.int32, device="cuda"))
        if own:
            import paper_2603_24239_b200 as dvm
            s["code"] = dvm.encode_paging(requests=n, max_blocks=width, page_size=page, rows=rows, free_pages=s["free"].numel())
        return s
    if case["op"] == "rotary":
        t, hq, hk, d, rot = case["tokens"], case["q_heads"], case["kv_heads"], case["dim"], case["rot"]
        rows, dt = t + case["pad"], BF16 if case["dtype"] == "bf16" else F32
        # the projections' output: one row of query, key and value heads per token
        qkv = _normal(g, (rows, hq + 2 * hk, d), dt)
        pages = _blocks(t, page) + 2
        table_rows = 16384
        first = host.randint(0, table_rows - t)
        positions = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        positions[:t] = torch.arange(first, first + t, device="cuda")
        slots = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        at = torch.randperm(pages, generator=g, device="cuda")
        k = torch.arange(t, device="cuda")
        slots[:t] = (at[k // page] * page + k % page).to(torch.int32)
        s.update(rows=rows, q=qkv[:, :hq], k=qkv[:, hq:hq + hk], v=qkv[:, hq + hk:], positions=positions, slots=slots,
                 wq=_normal(g, (d,), dt, 0.1, 1.0), wk=_normal(g, (d,), dt, 0.1, 1.0), angles=_angles(table_rows, rot), eps=1e-6,
                 q_out=torch.zeros((rows, hq, d), dtype=dt, device="cuda"),
                 k_cache=_normal(g, (pages, page, hk, d), dt), v_cache=_normal(g, (pages, page, hk, d), dt))
        if own:
            import paper_2603_24239_b200 as dvm
            s["code"] = dvm.encode_rotary(q=s["q"], k=s["k"], v=s["v"], angles=s["angles"], q_out=s["q_out"], k_cache=s["k_cache"],
                                          v_cache=s["v_cache"], wq=s["wq"] if case["norm"] else None, wk=s["wk"] if case["norm"] else None,
                                          eps=s["eps"], interleaved=case["interleaved"])
        return s
    cached, fresh = _lengths(case)
    n, hq, hk, d = case["requests"], case["q_heads"], case["kv_heads"], case["dim"]
    lengths, rows = cached + fresh, int(fresh.sum())
    blocks = _blocks(lengths, page)
    width, pages = int(blocks.max()), int(blocks.sum()) + 3
    pool = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(width, device="cuda")[None, :] < _ints(blocks)[:, None]] = pool[: int(blocks.sum())]
    shape = (pages, hk, page, d) if case["heads_first"] else (pages, page, hk, d)
    k_cache, v_cache = _normal(g, shape, BF16), _normal(g, shape, BF16)
    if case["heads_first"]:  # the same [page, token, head, dim] indices, other strides
        k_cache, v_cache = k_cache.transpose(1, 2), v_cache.transpose(1, 2)
    s.update(rows=rows, width=width, lengths=_ints(lengths), starts=_ints(np.concatenate([[0], np.cumsum(fresh)])), most=int(fresh.max()),
             q=_normal(g, (rows, hq, d), BF16, 1.3), k_cache=k_cache, v_cache=v_cache, table=table, scale=1.0 / math.sqrt(d),
             out=torch.zeros((rows, hq, d), dtype=BF16, device="cuda"))
    if own:
        import paper_2603_24239_b200 as dvm
        s["code"] = dvm.encode_attention(q=s["q"], k_cache=k_cache, v_cache=v_cache, table=table, out=s["out"], scale=s["scale"],
                                         window=case["window"], sinks=case["sinks"], max_q=s["most"])
        s["workspace"] = torch.empty(max(1, dvm.tensor_extents(s["code"])[-1]), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------- one pass

def run(s):
    return {"paging": _run_paging, "rotary": _run_rotary, "attention": _run_attention}[s["op"]](s)


def _run_paging(s):
    if own:
        import paper_2603_24239_b200 as dvm
        dvm.launch(s["code"], (s["cached"], s["new"], s["free"], s["table"], s["starts"], s["lengths"], s["positions"], s["slots"], s["taken"]))
        return {k: s[k] for k in ("table", "starts", "lengths", "positions", "slots", "taken")}
    page, rows, width, dev = s["page"], s["rows"], s["width"], s["table"].device
    cached, fresh = s["cached"].long(), s["new"].long()
    ends = fresh.cumsum(0)
    starts = torch.cat([ends.new_zeros(1), ends])
    held = (cached + page - 1) // page
    need = (cached + fresh + page - 1) // page - held
    before = need.cumsum(0) - need
    col = torch.arange(width, device=dev)[None, :]
    at = before[:, None] + col - held[:, None]
    is_new = (col >= held[:, None]) & (col < (held + need)[:, None])
    page_new = s["free"][at.clamp(0, s["free"].numel() - 1)]
    table = torch.where(is_new, torch.where(at < s["free"].numel(), page_new, -1), s["table"])
    t = torch.arange(rows, device=dev)
    req = torch.searchsorted(ends, t, right=True).clamp(max=s["requests"] - 1)
    pos = cached[req] + t - starts[req]
    block = (pos // page).clamp(0, width - 1)
    p = table[req, block].long()
    real = t < starts[-1]
    positions = torch.where(real, pos, -1).to(torch.int32)
    slots = torch.where(real & (p >= 0), p * page + pos % page, -1).to(torch.int32)
    return {"table": table, "starts": starts.to(torch.int32), "lengths": (cached + fresh).to(torch.int32), "positions": positions,
            "slots": slots, "taken": need.sum().to(torch.int32).reshape(1)}


def _turn(x, angles, positions, rot, interleaved):
    a = angles[positions.long()]
    c, sn = a[:, None, : rot // 2], a[:, None, rot // 2:]
    if interleaved:
        x1, x2 = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([x1 * c - x2 * sn, x2 * c + x1 * sn], -1).flatten(-2)
    else:
        x1, x2 = x[..., : rot // 2], x[..., rot // 2: rot]
        y = torch.cat([x1 * c - x2 * sn, x2 * c + x1 * sn], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _run_rotary(s):
    if own:
        import paper_2603_24239_b200 as dvm
        if s["norm"]:
            dvm.launch(s["code"], (s["q"], s["k"], s["v"], s["wq"], s["wk"], s["angles"], s["positions"], s["slots"], s["q_out"], s["k_cache"], s["v_cache"]))
        else:
            dvm.launch(s["code"], (s["q"], s["k"], s["v"], s["angles"], s["positions"], s["slots"], s["q_out"], s["k_cache"], s["v_cache"]))
        return {k: s[k] for k in ("q_out", "k_cache", "v_cache")}
    t = s["tokens"]  # the rows behind them are padding and stay as they are
    pos, slots = s["positions"][:t], s["slots"][:t].long()
    q, k = s["q"][:t].float(), s["k"][:t].float()
    if s["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + s["eps"]) * s["wq"].float()
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + s["eps"]) * s["wk"].float()
    dt = s["q_out"].dtype
    s["q_out"][:t] = _turn(q, s["angles"], pos, s["rot"], s["interleaved"]).to(dt)
    s["k_cache"].view(-1, s["kv_heads"], s["dim"])[slots] = _turn(k, s["angles"], pos, s["rot"], s["interleaved"]).to(dt)
    s["v_cache"].view(-1, s["kv_heads"], s["dim"])[slots] = s["v"][:t]
    return {k: s[k] for k in ("q_out", "k_cache", "v_cache")}


def _run_attention(s):
    if own:
        import paper_2603_24239_b200 as dvm
        dvm.launch(s["code"], (s["q"], s["k_cache"], s["v_cache"], s["table"], s["starts"], s["lengths"], s["out"], s["workspace"]))
        return s["out"]
    n, hq, hk, d, most, dev = s["requests"], s["q_heads"], s["kv_heads"], s["dim"], s["most"], s["q"].device
    starts, lengths = s["starts"].long(), s["lengths"].long()
    # keys and values of every request behind one another, padded to the longest
    at = s["table"].long().clamp(min=0)
    k = s["k_cache"][at].reshape(n, -1, hk, d).permute(0, 2, 3, 1).float()
    v = s["v_cache"][at].reshape(n, -1, hk, d).permute(0, 2, 1, 3).float()
    fresh = starts[1:] - starts[:-1]
    j = torch.arange(most, device=dev)
    row = (starts[:-1, None] + j[None, :]).clamp(max=s["rows"] - 1)
    q = s["q"][row].view(n, most, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(n, hk, -1, d).float()
    pos = (lengths - fresh)[:, None, None] + j[None, :, None]
    key = torch.arange(k.shape[-1], device=dev)[None, None, :]
    seen = (key <= pos) & (key < lengths[:, None, None])
    if s["window"]:
        seen &= (key > pos - s["window"]) | (key < s["sinks"])
    hidden = ~seen[:, None, None]
    w = torch.matmul(q, k).view(n, hk, hq // hk, most, -1).mul_(s["scale"]).masked_fill_(hidden, float("-inf"))
    w = w.sub_(w.amax(-1, keepdim=True).clamp_(min=torch.finfo(F32).min)).exp_()
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(n, hk, -1, w.shape[-1]), v).view(n, hk, hq // hk, most, d) / total.clamp(min=torch.finfo(F32).tiny)
    t = torch.arange(s["rows"], device=dev)
    req = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    return o.permute(0, 3, 1, 2, 4).reshape(n, most, hq, d)[req, t - starts[req]].to(BF16)


# ------------------------------------------------------------------------------------------------- exact values, work

def exact(case, seed):
    if case["op"] == "paging":
        return None
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "rotary":
        t, rot, half = case["tokens"], case["rot"], case["rot"] // 2
        ang = s["angles"].to(f64)[s["positions"][:t].long()]
        i = torch.arange(half, device="cuda")
        first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
        done = {}
        for part, weight in (("q", "wq"), ("k", "wk")):
            x = s[part][:t].to(f64).clone()
            if case["norm"]:
                x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / case["dim"] + s["eps"]) * s[weight].to(f64)
            z = torch.complex(x[..., first], x[..., second]) * torch.complex(ang[:, :half], ang[:, half:])[:, None]
            x[..., first], x[..., second] = z.real, z.imag
            done[part] = x
        out = {"q_out": s["q_out"].to(f64), "k_cache": s["k_cache"].to(f64), "v_cache": s["v_cache"].to(f64)}
        slot = s["slots"][:t].long()
        out["q_out"][:t] = done["q"]
        out["k_cache"][slot // case["page"], slot % case["page"]] = done["k"]
        out["v_cache"][slot // case["page"], slot % case["page"]] = s["v"][:t].to(f64)
        return out
    hq, hk, page = case["q_heads"], case["kv_heads"], case["page"]
    out = torch.zeros_like(s["out"], dtype=f64)
    cached, fresh = _lengths(case)
    row = 0
    for i in range(case["requests"]):
        total, new = int(cached[i] + fresh[i]), int(fresh[i])
        used = s["table"][i, : _blocks(total, page)].long()
        keys = s["k_cache"][used].flatten(0, 1)[:total].to(f64)
        vals = s["v_cache"][used].flatten(0, 1)[:total].to(f64)
        for h in range(hq):
            kh, vh = keys[:, h // (hq // hk)], vals[:, h // (hq // hk)]
            for b in range(0, new, 2048):
                m = min(2048, new - b)
                z = s["q"][row + b: row + b + m, h].to(f64) @ kh.T * s["scale"]
                p = torch.arange(total - new + b, total - new + b + m, device="cuda")[:, None]
                c = torch.arange(total, device="cuda")[None, :]
                off = c > p
                if case["window"]:
                    off |= (c + case["window"] <= p) & (c >= case["sinks"])
                out[row + b: row + b + m, h] = torch.softmax(z.masked_fill(off, -math.inf), -1) @ vh
        row += new
    return out


def work(case):
    page = case["page"]
    if case["op"] == "paging":
        cached, fresh = _lengths(case)
        new = int((_blocks(cached + fresh, page) - _blocks(cached, page)).sum())
        touched = int((_blocks(cached + fresh, page) - cached // page).sum())
        rows = int(fresh.sum()) + case["pad"]
        return {"bytes": 4 * (2 * len(cached) + new + touched + new + 2 * len(cached) + 2 + 2 * rows), "flops": 0}
    if case["op"] == "rotary":
        t, d, es = case["tokens"], case["dim"], 2 if case["dtype"] == "bf16" else 4
        values = t * (case["q_heads"] + 2 * case["kv_heads"]) * d
        return {"bytes": 2 * values * es + t * case["rot"] * 4 + 8 * (t + case["pad"]) + 2 * d * es, "flops": 8 * values}
    cached, fresh = _lengths(case)
    w, sinks = case["window"], case["sinks"]
    pairs = keys = 0
    for c, f in zip(cached.tolist(), fresh.tolist()):
        pos = np.arange(c, c + f, dtype=np.int64)
        if w:
            pairs += int((np.minimum(pos + 1, w) + np.minimum(sinks, np.maximum(0, pos + 1 - w))).sum())
            low = max(0, c - w + 1)
            keys += (c + f - low) + min(sinks, low)
        else:
            pairs += int((pos + 1).sum())
            keys += c + f
    rows = int(fresh.sum())
    return {"bytes": 2 * rows * case["q_heads"] * case["dim"] * 2 + 2 * keys * case["kv_heads"] * case["dim"] * 2 + 4 * int(_blocks(cached + fresh, page).sum()),
            "flops": 4 * pairs * case["q_heads"] * case["dim"]}
