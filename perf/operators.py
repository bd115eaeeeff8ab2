"""The operators of token streams that are timed, and how a program calls them.

Three operators, in the directions in which they are used:

  how = "serve"   product of tokens with a weight matrix held in 8 bits: every token gets a scale of its own when it
                  arrives, every output channel has had one since the weights were laid out;
  how = "train"   the same product with both gradients, from weights in floating point: codes with stochastic rounding
                  for the gradients, the scales of the summed axis folded in before the codes are made;
  how = "cache"   keys and values quantised as they are written into a paged cache (a scale for each token and head),
                  and read back;
  how = "attend"  attention of the newest tokens of each request over its pages of that cache: single tokens, chunks of a
                  prompt, or another sequence's states (not causal).

The arithmetic that decides a code is fp32, each operation rounded once: c = max|x|, inv = 127 / c, code = rint(x * inv),
scale = c / 127; with stochastic rounding |code| = floor((|x| * (inv * 2^24) + u) / 2^24), u 24 bits of (seed, index).
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SEED = 20                      # of the stochastic rounding: every backward pass with the same draws


def _linear(name, how, M, K, N, dtype, bias):
    c = dict(how=how, M=M, K=K, N=N, dtype=dtype, bias=bias)
    return dict(c, name=name) if name else c


def _cache(name, tokens, back, heads, dim, page, dtype, skip=0):
    c = dict(how="cache", tokens=tokens, back=back, heads=heads, dim=dim, page=page, dtype=dtype, skip=skip)
    return dict(c, name=name) if name else c


def _attend(name, B, new, new_least, most, least, heads, group, dim, page, dtype, causal=True, shape=1):
    """B requests of new_least .. new new tokens and least .. most cached ones (the new ones among them where causal)."""
    c = dict(how="attend", B=B, new=new, new_least=new_least, most=most, least=least, heads=heads, group=group, dim=dim,
             page=page, dtype=dtype, causal=causal, shape=shape)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a projection of one token while text is generated: latency, the weights read once
        _linear("serve_1", "serve", 1, 4096, 4096, "bf16", False),
        # a handful of requests through a classifier of odd width
        _linear("serve_9_odd", "serve", 9, 2048, 1000, "f16", True),
        # an odd chunk of a prompt through a widening layer
        _linear("serve_chunk_1001", "serve", 1001, 4096, 16384, "f16", True),
        # long prompts together: as much arithmetic as a serving program sees in one call
        _linear("serve_16384", "serve", 16384, 4096, 4096, "bf16", False),
        # a training pass of the classifier 2048 -> 1000 at batch 256
        _linear("train_fc", "train", 256, 2048, 1000, "f32", True),
        # a training pass of a square projection over 8192 tokens
        _linear("train_8192", "train", 8192, 4096, 4096, "bf16", False),
        # one new token for each of 64 requests, and one request's 509 tokens handed to another program
        _cache("cache_step", 64, 509, 8, 128, 16, "bf16"),
        # a long prompt written and read back, some of its tokens without a place
        _cache("cache_prompt", 16384, 16384, 8, 128, 64, "f16", skip=37),
        # one request's next token
        _attend("attend_1", 1, 1, 1, 1021, 1021, 8, 4, 128, 16, "bf16"),
        # the next token of 64 requests of very different lengths
        _attend("attend_64_requests", 64, 1, 1, 8192, 1, 8, 4, 128, 16, "bf16", shape=2),
        # the last chunk of two long prompts
        _attend("attend_chunk", 2, 2048, 2048, 8192, 8000, 8, 4, 128, 64, "bf16", shape=3),
        # another sequence's states, nine ragged requests in fp32, some of them empty, pages of 24 tokens
        _attend("attend_states_f32", 9, 131, 1, 1500, 0, 12, 1, 64, 24, "f32", causal=False, shape=4),
    ]


def _lengths(c):
    """New and cached tokens of each request: of the case alone."""
    rng = random.Random(c["shape"])
    new, have = [], []
    for _ in range(c["B"]):
        n = rng.randint(c["new_least"], c["new"])
        new.append(n)
        have.append(max(rng.randint(c["least"], c["most"]), n if c["causal"] else 0))
    if c["B"] > 1:
        have[0] = max(c["most"], have[0])
        if not c["least"]:
            have[-1] = 0 if not c["causal"] else have[-1]
    return new, have


def work(c):
    """What a pass cannot do without: inputs read once, outputs written once, two operations for each multiplication and addition."""
    if c["how"] in ("serve", "train"):
        M, K, N = c["M"], c["K"], c["N"]
        e = 4 if c["dtype"] == "f32" else 2
        if c["how"] == "serve":
            return {"bytes": e * M * (K + N) + N * K + 4 * N * (2 if c["bias"] else 1), "flops": 2 * M * N * K}
        return {"bytes": e * (2 * M * K + 2 * N * K + 2 * M * N), "flops": 6 * M * N * K}
    e = 4 if c["dtype"] == "f32" else 2
    row = c["heads"] * c["dim"]
    if c["how"] == "cache":
        return {"bytes": 2 * (c["tokens"] + c["back"]) * (row * (e + 1) + 4 * c["heads"]), "flops": 8 * (c["tokens"] + c["back"]) * row}
    new, have = _lengths(c)
    pairs = sum(sum(max(0, h - n + 1 + i) for i in range(n)) if c["causal"] else n * h for n, h in zip(new, have))
    return {"bytes": sum(2 * h * (row + 4 * c["heads"]) for h in have) + 2 * e * sum(new) * row * c["group"],
            "flops": 4 * pairs * row * c["group"]}


def _most():
    by = {}
    for c in listed():
        w = work(c)
        b, f = by.get(c["how"], (0, 0))
        by[c["how"]] = max(b, w["bytes"]), max(f, w["flops"])
    return by


def draw(rng):
    most = _most()

    def log_int(lo, hi):
        return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))

    while True:
        how = rng.choice(["serve", "train", "cache", "attend", "attend"])
        dtype = rng.choice(["f32", "bf16", "f16"])
        if how in ("serve", "train"):
            K, N = log_int(256, 8192), log_int(200, 16384)
            if rng.random() < 0.7:
                K = -(-K // 64) * 64
            if rng.random() < 0.5:
                N = -(-N // 64) * 64
            c = _linear(None, how, log_int(1, 16384) if how == "serve" else log_int(64, 8192), K, N, dtype, rng.random() < 0.5)
            if 3072 in (c["M"], c["K"], c["N"]):
                continue
        elif how == "cache":
            c = _cache(None, log_int(1, 16384), log_int(1, 16384), rng.choice([1, 2, 4, 8, 12]), rng.choice([64, 80, 96, 128, 256]),
                       rng.choice([1, 16, 24, 32, 64, 128]), dtype, rng.choice([0, 0, 5]))
        else:
            dim = rng.choice([64, 80, 96, 128, 128, 256])
            heads, group = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 2, 3, 4, 7, 8, 16])
            new = 1 if rng.random() < 0.4 else log_int(2, 2048)
            longest = log_int(16, 16384)
            causal = rng.random() < 0.75
            c = _attend(None, log_int(1, 64), new, rng.choice([1, new]), max(longest, new), rng.choice([0, 1, longest // 2]),
                        heads, group, dim, rng.choice([1, 16, 24, 32, 64, 128]), dtype, causal, rng.randrange(1 << 20))
            # what a plain form holds: padded scores, and keys and values in 32 bits
            if c["B"] * c["new"] * c["most"] * heads * group > 1.2e9 or c["B"] * c["most"] * heads * dim > 6e8:
                continue
        w = work(c)
        if w["bytes"] <= most[how][0] and w["flops"] <= most[how][1]:
            return c


def _codes_of(x):
    """Codes and scales of the last axis, nearest rounding."""
    x = x.float()
    c = x.abs().amax(-1, keepdim=True)
    inv = torch.where(c > 0, torch.full_like(c, 127.0) / c, torch.zeros_like(c))
    return torch.clamp(x * inv, -127.0, 127.0).round(), torch.where(c > 0, c / 127.0, torch.zeros_like(c))


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[c["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    state = dict(c)
    if c["how"] in ("serve", "train"):
        M, K, N = c["M"], c["K"], c["N"]
        # a token's values spread over a few channels that are much larger than the others, and tokens differ in size
        x = normal(M, K) * torch.exp(0.5 * normal(M, 1))
        x = x * torch.where(torch.rand(K, generator=gen, device="cuda") < 0.005, 10.0, 1.0)
        state["x"] = x.to(dt)
        w = normal(N, K) * (1.0 / math.sqrt(K)) * torch.exp(0.3 * normal(N, 1))
        b = normal(N) * 0.1 if c["bias"] else None
        if c["how"] == "train":
            g = normal(M, N) * 1e-3 * torch.exp(normal(M, 1))
            state.update(x=state["x"].requires_grad_(True), w=w.to(dt).requires_grad_(True), g=g.to(dt),
                         b=None if b is None else b.requires_grad_(True))
            return state
        q, s = _codes_of(w)
        # rows of codes lie 16 bytes apart or a multiple of it, zeros between them
        wq = torch.zeros(N, -(-K // 16) * 16, dtype=torch.int8, device="cuda")
        wq[:, :K] = q
        state.update(wq=wq, sw=s[:, 0].contiguous(), b=b)
        if own:
            from paper_1912_12607_amd import tokens
            state["layer"] = tokens.ServedLinear(wq, state["sw"], K, state["b"])
        return state
    H, D, page = c["heads"], c["dim"], c["page"]
    host = random.Random(seed)
    if c["how"] == "cache":
        T, R = c["tokens"], c["back"]
        pages = -(-2 * (T + R) // page) + 1
        order = torch.randperm(pages * page, generator=gen, device="cuda")
        slots = order[:T].clone()
        if c["skip"]:
            slots[::c["skip"]] = -1                     # tokens of requests that are gone
        # what is read back: the tokens written, and as far as they do not reach, others
        back = torch.cat([slots, order[T:]])[:R].clone()
        live = torch.arange(T, device="cuda")
        state["live"] = live[live % c["skip"] != 0] if c["skip"] else live
        state.update(k=(normal(T, H, D) * torch.exp(normal(T, H, 1))).to(dt), v=normal(T, H, D).to(dt), slots=slots, back_slots=back)
    else:
        new, have = _lengths(c)
        B, T = c["B"], sum(new)
        need = [-(-h // page) for h in have]
        pages = sum(need) + 3
        ids = list(range(pages))
        host.shuffle(ids)
        width = max(1, max(need))
        table = [[0] * width for _ in range(B)]
        for b, n in enumerate(need):
            table[b][:n] = [ids.pop() for _ in range(n)]
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        dev = dict(dtype=torch.int32, device="cuda")
        state.update(q=(normal(T, H * c["group"], D) * 1.5).to(dt), starts=torch.tensor(starts, **dev), lengths=torch.tensor(have, **dev),
                     table=torch.tensor(table, **dev), new_most=max(new), longest=max(have))
    shape = (pages, H, page)
    for name in ("k", "v"):
        state[name + "q"] = torch.randint(-127, 128, shape + (D,), generator=gen, device="cuda", dtype=torch.int8)
        state[name + "s"] = torch.exp(0.4 * normal(*shape)) * (1.0 / 64)
    if own:
        from paper_1912_12607_amd import tokens
        state["cache"] = tokens.PagedCache(state["kq"], state["ks"], state["vq"], state["vs"])
    return state


# The stochastic draw of an element: two keys from the seed, one hash over its index (64-bit integers, the low 32 bits kept).
_LOW = 0xFFFFFFFF


def _mix(x):
    x = x ^ (x >> 16)
    x = (x * 0x85EBCA6B) & _LOW
    x = x ^ (x >> 13)
    x = (x * 0xC2B2AE35) & _LOW
    return x ^ (x >> 16)


def _stochastic_codes(x, axis, seed):
    """Codes of fp32 x with a scale for each slice across `axis`; the index of an element is its place in x."""
    kx = _mix((seed & _LOW) ^ _mix(((seed >> 32) + 0x9E3779B9) & _LOW))
    ka = _mix((kx + 0x9E3779B9) & _LOW)
    i = torch.arange(x.numel(), device=x.device).view(x.shape)
    u = _mix(((i ^ kx) + ka) & _LOW) >> 8
    c = x.abs().amax(axis, keepdim=True)
    inv = torch.where(c > 0, torch.full_like(c, 127.0) / c, torch.zeros_like(c)) * 16777216.0
    # the sum of product and draw is needed exactly: 64 bits
    m = torch.floor((x.abs().double() * inv.double() + u.double()) / 16777216.0).clamp(max=127.0).float()
    return torch.where(x < 0, -m, m), torch.where(c > 0, c / 127.0, torch.zeros_like(c))


def run(state):
    how, dt = state["how"], DTYPES[state["dtype"]]
    if how == "serve":
        if own:
            return state["layer"](state["x"])
        xq, sx = _codes_of(state["x"])
        y = torch.matmul(xq, state["wq"][:, :state["K"]].float().t()) * (sx * state["sw"])
        return (y if state["b"] is None else y + state["b"]).to(dt)
    if how == "train":
        x, w, g, b = state["x"], state["w"], state["g"], state["b"]
        if own:
            from paper_1912_12607_amd import tokens
            y = tokens.linear(x, w, b, seed=SEED)
            grads = torch.autograd.grad(y, [x, w] if b is None else [x, w, b], g)
            return {"y": y.detach(), "dx": grads[0], "dw": grads[1], **({} if b is None else {"db": grads[2]})}
        with torch.no_grad():
            xq, sx = _codes_of(x)
            wq, sw = _codes_of(w)
            y = torch.matmul(xq, wq.t()) * (sx * sw.t())
            g32 = g.float()
            gq, sg = _stochastic_codes(g32 * sw.t(), 1, SEED)
            dx = torch.matmul(gq, wq) * sg
            hq, sh = _stochastic_codes(g32 * sx, 0, SEED ^ (1 << 63))
            dw = torch.matmul(hq.t(), xq) * sh.t()
            out = {"y": (y if b is None else y + b).to(dt), "dx": dx.to(dt), "dw": dw.to(dt)}
            return out if b is None else dict(out, db=g32.sum(0))
    if how == "cache":
        if own:
            state["cache"].write(state["k"], state["v"], state["slots"])
            k, v = state["cache"].read(state["back_slots"], dt)
            return {"k": k, "v": v, "ks": state["ks"], "vs": state["vs"]}
        out, page = {}, state["page"]
        live = state["live"]                             # the tokens that have a place
        p, o = torch.div(state["slots"][live], page, rounding_mode="floor"), state["slots"][live] % page
        at = state["back_slots"].clamp(min=0)
        rp, ro = torch.div(at, page, rounding_mode="floor"), at % page
        for name in ("k", "v"):
            codes, s = _codes_of(state[name])
            q, sc = state[name + "q"], state[name + "s"]
            q[p, :, o] = codes[live].to(torch.int8)
            sc[p, :, o] = s[live][..., 0]
            back = q[rp, :, ro].float() * sc[rp, :, ro][..., None]
            out[name] = torch.where((state["back_slots"] >= 0)[:, None, None], back, torch.zeros_like(back)).to(dt)
            out[name + "s"] = sc
        return out
    if own:
        return state["cache"].attend(state["q"], state["starts"], state["lengths"], state["table"], causal=state["causal"],
                                     longest=state["longest"])
    return _attend_plain(state).to(dt)


def _attend_plain(s):
    """Keys and values of each request side by side, in fp32; scores, softmax and sums over the padded length."""
    B, H, G, D, n, L = s["B"], s["heads"], s["group"], s["dim"], s["new_most"], s["table"].shape[1] * s["page"]
    T = s["q"].shape[0]
    dev = s["q"].device
    ids, lengths, starts = s["table"].long(), s["lengths"].long(), s["starts"].long()
    new = starts[1:] - starts[:-1]
    j = torch.arange(L, device=dev)
    there = j < lengths[:, None]                                                            # B, L

    def gathered(q, sc):
        x = q[ids].permute(0, 2, 1, 3, 4).reshape(B, H, L, D).float()
        x *= sc[ids].permute(0, 2, 1, 3).reshape(B, H, L, 1)
        return x.masked_fill_(~there[:, None, :, None], 0.0)

    i = torch.arange(n, device=dev)
    at = (starts[:-1, None] + i).clamp(max=max(T - 1, 0))                                   # B, n
    q = s["q"][at].float().view(B, n, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, D)
    scores = torch.matmul(q, gathered(s["kq"], s["ks"]).transpose(2, 3)).view(B, H, G, n, L).mul_(1.0 / math.sqrt(D))
    seen = there[:, None, :].expand(B, n, L)
    if s["causal"]:
        seen = seen & (j <= (lengths - new)[:, None, None] + i[:, None])
    scores.masked_fill_(~seen[:, None, None], float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores.sub_(torch.where(top == float("-inf"), torch.zeros_like(top), top)))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, H, G * n, L), gathered(s["vq"], s["vs"])).view(B, H, G, n, D)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    t = torch.arange(T, device=dev)
    b = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    return out[b, :, :, t - starts[b]].reshape(T, H * G, D)


def exact(c, seed):
    """The definitions in 64 bits: what rounds in fp32 by definition (the codes) is formed in 64 bits and rounded there."""
    s = prepare(c, seed)
    f64, f32 = torch.float64, torch.float32

    def once(v):
        return v.to(f32).to(f64)

    def scales(v, axis):
        top = v.abs().amax(axis, keepdim=True)
        safe = torch.where(top == 0, torch.ones_like(top), top)
        return torch.where(top == 0, 0 * top, once(127.0 / safe)), torch.where(top == 0, 0 * top, once(top / 127.0))

    def nearest(v, axis=-1):
        inv, sc = scales(v, axis)
        return torch.round(once(v * inv)).clamp(-127, 127), sc

    def to_plus(v, axis, key):
        """floor(|v| / scale + draw), the draw a multiple of 2^-24."""
        def h(a):
            for shift, by in ((16, 0x85EBCA6B), (13, 0xC2B2AE35)):
                a = ((a ^ (a >> shift)) * by) % (1 << 32)
            return a ^ (a >> 16)
        first = h((key % (1 << 32)) ^ h((key // (1 << 32) + 0x9E3779B9) % (1 << 32)))
        second = h((first + 0x9E3779B9) % (1 << 32))
        index = torch.arange(v.numel(), device=v.device).reshape(v.shape)
        draws = (h(((index ^ first) + second) % (1 << 32)) // 256).to(f64) / 2.0**24
        inv, sc = scales(v, axis)
        return torch.sign(v) * torch.clamp(torch.floor(v.abs() * inv + draws), max=127), sc

    if c["how"] == "serve":
        q, sx = nearest(s["x"].to(f64))
        y = (q @ s["wq"][:, :c["K"]].to(f64).T) * sx * s["sw"].to(f64)
        return y if s["b"] is None else y + s["b"].to(f64)
    if c["how"] == "train":
        x, w, g = (s[k].detach().to(f64) for k in ("x", "w", "g"))
        (xq, sx), (wq, sw) = nearest(x), nearest(w)
        y = xq @ wq.T * sx * sw.T
        a, sa = to_plus(once(g * sw.T), 1, SEED)
        b, sb = to_plus(once(g * sx), 0, SEED + (1 << 63))
        out = {"y": y if s["b"] is None else y + s["b"].detach().to(f64), "dx": a @ wq * sa, "dw": (b.T @ xq) * sb.T}
        return out if s["b"] is None else dict(out, db=g.sum(0))
    if c["how"] == "cache":
        out = {}
        page = c["page"]
        for name in ("k", "v"):
            q, sc = s[name + "q"].to(f64), s[name + "s"].to(f64)
            codes, sn = nearest(s[name].to(f64))
            live = torch.nonzero(s["slots"] >= 0).flatten()
            to = s["slots"][live]
            q[to // page, :, to % page] = codes[live]
            sc[to // page, :, to % page] = sn[live].squeeze(-1)
            at = s["back_slots"]
            back = torch.zeros(c["back"], c["heads"], c["dim"], dtype=f64, device=q.device)
            have = torch.nonzero(at >= 0).flatten()
            back[have] = q[at[have] // page, :, at[have] % page] * sc[at[have] // page, :, at[have] % page].unsqueeze(-1)
            out[name], out[name + "s"] = back, sc
        return out
    new, have = _lengths(c)
    page, D, G = c["page"], c["dim"], c["group"]
    out = torch.zeros(s["q"].shape, dtype=f64, device=s["q"].device)
    at = 0
    for b, (n, h) in enumerate(zip(new, have)):
        if n and h:
            ids = s["table"][b, :-(-h // page)].long()
            for head in range(c["heads"]):
                k, v = ((s[m + "q"][ids, head].to(f64) * s[m + "s"][ids, head].to(f64).unsqueeze(-1)).reshape(-1, D)[:h] for m in ("k", "v"))
                q = s["q"][at:at + n, head * G:(head + 1) * G].to(f64).reshape(n * G, D)
                a = (q @ k.T) / math.sqrt(D)
                if c["causal"]:
                    last = h - n + torch.arange(n, device=q.device).repeat_interleave(G)
                    a = a.masked_fill(torch.arange(h, device=q.device) > last[:, None], float("-inf"))
                out[at:at + n, head * G:(head + 1) * G] = (torch.softmax(a, -1) @ v).reshape(n, G, D)
        at += n
    return out
