"""Performance cases of what stands around a layer's compression: positions,
the prompt's attention, and a cache of the kept rows in 4 bits.

  rotate   rotary positions of a projection's queries and keys, at the end of
           which they are what compression, cache and attention take: half and
           interleaved layouts, part of the head, three rows of positions for
           images and video, frequencies scaled for long contexts, the heads
           normalised first where the model does
  prompt   causal attention of a ragged batch of prompts, or of their next
           chunks over the rows before them, with the normalisers of the window
           rows that the compression reads
  store    the kept rows gathered and quantised to 4 bits (e2m1, a power-of-two
           scale for every 32 values of a row), and read back
  step     a decode step of one layer over such a cache: the new tokens' rows
           appended, attention, the drafted tokens then rolled back; the rows
           appended are returned
  attend   attention over such a cache alone

`run` computes each in elementary torch operations, or with the framework's
calls where `own` is set.  A pair is a (layer, sequence, KV head).
"""
from __future__ import annotations

import math

import torch

own = False

GROUP, E_LOW, E_HIGH = 32, -100, 125      # values of a scale, exponents it may take
RESERVE = 64
LARGEST_ROWS = 300_000_000                # values of K held by a drawn cache, padded
LARGEST_LOGITS = 1_900_000_000            # logits of a drawn prompt, padded
LARGEST_TURNED = 160_000_000              # values of a drawn rotation
NORM_EPS = 1e-6


def _case(name, **c):
    return dict(name=name, **c) if name else c


def _rotate(name, tokens, hq, hkv, d, rotary, dtype, layout="half", sections="", base=1e4, scaling="plain",
            factor=1.0, trained=0, norm=False, far=0):
    """`far`: the first position (a token decoded behind a long prompt)."""
    return _case(name, op="rotate", tokens=tokens, hq=hq, hkv=hkv, d=d, rotary=rotary, dtype=dtype, layout=layout,
                 sections=sections, base=base, scaling=scaling, factor=factor, trained=trained, norm=norm, far=far)


def _prompt(name, hq, hkv, d, window, dtype, lens, queries=None):
    """`queries`: the last so many tokens of each prompt are this call's chunk."""
    return _case(name, op="prompt", hq=hq, hkv=hkv, d=d, window=window, dtype=dtype, lens=",".join(map(str, lens)),
                 queries=",".join(map(str, queries or lens)))


def _kept(name, op, layers, hq, hkv, d, window, bt, dtype, lens, budgets, new=1, whole=False, counts=False):
    return _case(name, op=op, layers=layers, hq=hq, hkv=hkv, d=d, window=window, bt=bt, dtype=dtype,
                 lens=",".join(map(str, lens)), budgets=",".join(map(str, budgets)), new=new, whole=whole,
                 counts=counts)


def listed():
    ragged = (9631, 5167, 14011, 1291, 3083, 11117, 7411, 2049)
    chunks = (512, 512, 512, 512, 11, 512, 1, 257)
    many = tuple(900 + (i * 2377) % 7001 for i in range(64))
    mbud = tuple((64, 128, 512)[i % 3] for i in range(64))
    return [
        # one new token of a model with images, far behind its prompt: latency
        _rotate("rotate-token", 1, 28, 4, 128, 128, "bf16", sections="16,24,24", base=1e6, far=8192),
        # an odd number of tokens in full precision, a quarter of the head turned in pairs
        _rotate("rotate-pairs-fp32", 4099, 14, 2, 64, 16, "fp32", layout="pairs", base=1e4),
        # the headline prompt's projection: normalised heads, a context scaled to four times its length
        _rotate("rotate-video-32k", 32768, 32, 8, 128, 128, "bf16", base=1e6, scaling="yarn", factor=4.0,
                trained=8192, norm=True),
        # the smallest prompt, in full precision: latency
        _prompt("prompt-tiny-fp32", 4, 4, 64, 8, "fp32", (512,)),
        # a prompt whose query heads have KV heads of their own
        _prompt("prompt-mha-2k", 32, 32, 128, 32, "bf16", (2048,)),
        # a prompt of images: matrix instructions
        _prompt("prompt-gqa-8k", 28, 4, 128, 32, "bf16", (8192,)),
        # a ragged batch whose prompts come in chunks, one of them a single token
        _prompt("prompt-chunks-b8", 32, 8, 128, 32, "bf16", ragged, chunks),
        # the headline prompt: 256 + 32 of 32K rows of every head and layer
        _kept("store4-video-32k", "store", 32, 32, 8, 128, 32, 64, "bf16", (32768,), (256,)),
        # one token of 16 sequences, every query head with a KV head of its own
        _kept("step4-mha-b16", "step", 1, 32, 32, 128, 32, 16, "bf16", (2048,) * 16,
              tuple(64 + 37 * i for i in range(16)), whole=True),
        # up to four drafted tokens of 64 sequences
        _kept("step4-drafts-b64", "step", 1, 28, 4, 128, 32, 32, "bf16", many, mbud, new=4, whole=True, counts=True),
        # full precision, a small-head model, five tokens of four sequences
        _kept("attend4-fp32-n5", "attend", 1, 14, 2, 64, 16, 32, "fp32", (4099, 12289, 777, 8191),
              (4083, 12273, 761, 8175), new=5, whole=True),
        # a prompt of 128K tokens kept whole: one sequence over the whole GPU
        _kept("attend4-128k", "attend", 1, 32, 8, 128, 32, 64, "bf16", (131072,), (131040,), whole=True),
    ]


HEADS = ((4, 4), (32, 32), (28, 4), (32, 8), (14, 2), (32, 1), (64, 8))


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def around(mid, lo, hi, n):
        return tuple(max(lo, min(hi, int(mid * math.exp(rng.uniform(-0.7, 0.7))))) for _ in range(n))

    while True:
        op = rng.choice(("rotate", "rotate", "prompt", "prompt", "prompt", "store", "step", "attend"))
        hq, hkv = rng.choice(HEADS)
        d, dtype = rng.choice((64, 128, 128)), rng.choice(("bf16", "bf16", "bf16", "fp32"))
        window = rng.choice((1, 8, 16, 32))
        if op == "rotate":
            tokens = log_int(1, 32768)
            rotary = rng.choice((d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)))
            a = rng.randint(0, rotary // 2)
            b = rng.randint(0, rotary // 2 - a)
            sections = rng.choice(("", "%d,%d,%d" % (a, b, rotary // 2 - a - b)))
            scaling = rng.choice(("plain", "linear", "ntk", "yarn"))
            if scaling == "ntk" and rotary < 4 or tokens * (hq + hkv) * d > LARGEST_TURNED:
                continue
            return _rotate(None, tokens, hq, hkv, d, rotary, dtype, rng.choice(("half", "pairs")), sections,
                           rng.choice((1e4, 5e5, 1e6)), scaling, 1.0 if scaling == "plain" else rng.choice((2.0, 4.0, 8.0)),
                           8192 if scaling == "yarn" else 0, rng.random() < 0.4, log_int(1, 131072) - 1)
        batch = log_int(1, 64)
        if op == "prompt":
            batch = log_int(1, 16)
            lens = around(log_int(1, 32768), 1, 32768, batch)
            queries = lens if rng.random() < 0.5 else tuple(min(n, m) for n, m in zip(lens, around(log_int(1, 2048), 1, 2048, batch)))
            if batch * hq * max(queries) * max(lens) > LARGEST_LOGITS // (2 if dtype == "fp32" else 1):
                continue
            return _prompt(None, hq, hkv, d, window, dtype, lens, queries)
        bt = rng.choice((16, 32, 64))
        layers = log_int(1, 32) if op == "store" else 1
        new = rng.choice((1, 1, 1, 2, 3, 5, 8)) if op != "store" else 1
        if hq // hkv * new > 64:
            continue
        top = {"store": 32768, "step": 8192, "attend": 131072}[op]
        lens = around(log_int(window + 1, top), window, top, batch)
        whole = op != "store" or rng.random() < 0.3
        if op == "attend" or whole and rng.random() < 0.5:
            budgets = tuple(max(1, n - window) for n in lens)
        else:
            budgets = tuple(max(1, min(n - window, log_int(16, 1024))) for n in lens)
        rows = max(min(k, n - window) + window for k, n in zip(budgets, lens))
        if layers * batch * hkv * rows * d > LARGEST_ROWS or layers * sum(lens) * hkv * d > LARGEST_ROWS:
            continue
        return _kept(None, op, layers, hq, hkv, d, window, bt, dtype, lens, budgets, new, whole,
                     new > 1 and batch > 1 and rng.random() < 0.5)


def _ints(s):
    return tuple(int(x) for x in s.split(",")) if s else ()


def _most_rows(case):
    return max(min(k, n - case["window"]) + case["window"]
               for k, n in zip(_ints(case["budgets"]), _ints(case["lens"])))


# ---- inputs

def _positions(case, g):
    """Text counts on; with three rows of positions a span of the prompt lies on a
    grid of frames, rows and columns, as images and video do."""
    n, far = case["tokens"], case["far"]
    p = torch.arange(n, device="cuda") + far
    if not case["sections"]:
        return p.int()
    side = 32
    i = torch.arange(n, device="cuda")
    grid = torch.stack([far + i // (side * side), far + i // side % side, far + i % side])
    image = (i >= n // 16) & (i < n - n // 8)
    return torch.where(image, grid, p).int()


def _rnd(seed):
    g = torch.Generator(device="cuda").manual_seed((seed * 1000003 + 31) & 0x7FFFFFFF)
    return g, lambda *s: torch.randn(*s, device="cuda", generator=g)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _projection(case, rnd, *tokens):
    """A fused projection's output [.., hq + 2 hkv, d]: unit-variance keys with a
    few strong channels, queries somewhat larger."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    x = rnd(*tokens, hq + 2 * hkv, d)
    x[..., :hq, :] *= 1.3
    x[..., hq:hq + hkv, :] *= torch.where(torch.arange(d, device="cuda") % 61 == 7, 4.0, 1.0)
    return x


def _split(case, x):
    hq, hkv = case["hq"], case["hkv"]
    return x[..., :hq, :], x[..., hq:hq + hkv, :], x[..., hq + hkv:, :]


def _inputs(case, seed):
    g, rnd = _rnd(seed)
    dt, dev, st = _dtype(case), dict(device="cuda"), dict(op=case["op"], case=case)
    if case["op"] == "rotate":
        st["q"], st["k"], _ = _split(case, _projection(case, rnd, case["tokens"]).to(dt))
        st["positions"] = _positions(case, g)
        st["q_norm"] = (1.0 + 0.2 * rnd(case["d"])).to(dt) if case["norm"] else None
        st["k_norm"] = (1.0 + 0.2 * rnd(case["d"])).to(dt) if case["norm"] else None
        return st
    lens = _ints(case["lens"])
    B = len(lens)
    cu = torch.tensor([0] + list(lens)).cumsum(0).tolist()
    st.update(cu=cu, cu_t=torch.tensor(cu, dtype=torch.int64, **dev), len_t=torch.tensor(lens, dtype=torch.int64, **dev))
    if case["op"] == "prompt":
        queries = _ints(case["queries"])
        st["cuq"] = torch.tensor([0] + list(queries)).cumsum(0).tolist()
        st["cuq_t"] = torch.tensor(st["cuq"], dtype=torch.int64, **dev)
        x = _projection(case, rnd, cu[-1])
        x[st["cu_t"][:-1], case["hq"]:case["hq"] + case["hkv"]] *= 2.0         # the sink: a strong first key
        q, st["k"], st["v"] = _split(case, x.to(dt))
        st["q"] = q
        if queries != lens:                                                   # the chunk's own projection
            at = torch.cat([torch.arange(cu[b + 1] - n, cu[b + 1], **dev) for b, n in enumerate(queries)])
            st["q"] = _split(case, x.to(dt)[at])[0]
        return st
    L, hkv, d, W, n = case["layers"], case["hkv"], case["d"], case["window"], case["new"]
    budgets = _ints(case["budgets"])
    st["K"] = torch.tensor(budgets, dtype=torch.int32, **dev)
    need = sum(L * hkv * -(-(min(k, m - W) + W + RESERVE) // case["bt"]) for k, m in zip(budgets, lens))
    st["blocks"] = need + 3
    st["free"] = torch.randperm(st["blocks"], device="cuda", generator=g).int()
    channel = torch.where(torch.arange(d, **dev) % 61 == 7, 4.0, 1.0)
    k = torch.empty(L, cu[-1], hkv, d, dtype=dt, **dev)
    v = torch.empty_like(k)
    for layer in range(L):
        kk = rnd(cu[-1], hkv, d)
        kk[st["cu_t"][:-1]] *= 2.0
        k[layer] = kk * channel
        v[layer] = rnd(cu[-1], hkv, d)
    st["k"], st["v"] = k, v
    if case["op"] == "store" and not case["whole"]:
        per = []
        for b in range(B):
            m = lens[b] - W
            kept = min(budgets[b], m)
            at = torch.rand(L, hkv, max(1, m), device="cuda", generator=g)[..., :m].topk(kept, -1).indices
            at = at.sort(-1).values.int()
            pad = torch.full((L, hkv, budgets[b] - kept), -1, dtype=torch.int32, **dev)
            per.append(torch.cat([at, pad], -1).reshape(L, -1))
        st["idx"] = torch.cat(per, 1).contiguous()
    if case["op"] in ("step", "attend"):
        st["q"], st["k_new"], st["v_new"] = _split(case, _projection(case, rnd, B, n).to(dt))
        st["counts"] = torch.randint(0, n + 1, (B,), dtype=torch.int32, device="cuda", generator=g) if case["counts"] else None
        st["back"] = torch.full((B,), -n, dtype=torch.int32, **dev) if st["counts"] is None else -st["counts"]
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    op = case["op"]
    if own:
        from paper_2606_14782_amd import bacon
        st["bacon"] = bacon
    if op == "rotate":
        if own:
            st["rotary"] = bacon.Rotary(
                case["hq"], case["hkv"], case["d"], case["dtype"], case["rotary"],
                layout={"half": bacon.ROTARY_HALF, "pairs": bacon.ROTARY_PAIRS}[case["layout"]],
                sections=_ints(case["sections"]) or None, base=case["base"],
                scaling={"plain": bacon.ROTARY_PLAIN, "linear": bacon.ROTARY_LINEAR, "ntk": bacon.ROTARY_NTK,
                         "yarn": bacon.ROTARY_YARN}[case["scaling"]],
                factor=case["factor"], trained_tokens=case["trained"], norm_eps=NORM_EPS)
        else:
            st["freq"], st["magnitude"] = _frequencies(case)
        return st
    if op == "prompt":
        if own:
            lens = _ints(case["lens"])
            st["shape"] = bacon.Shape(1, case["hq"], case["hkv"], case["d"], case["window"], len(lens), st["cu"][-1],
                                      bacon.BF16 if case["dtype"] == "bf16" else bacon.FP32)
            st["batch"] = bacon.BatchLayout(st["cu"], [1] * len(lens))
        return st
    st["most"] = _most_rows(case)
    bt = case["bt"]
    if own:
        lens, budgets = _ints(case["lens"]), _ints(case["budgets"])
        st["batch"] = bacon.BatchLayout(st["cu"], budgets)
        st["cache"] = bacon.Cache(case["layers"], case["hq"], case["hkv"], case["d"], case["window"], bt, len(lens),
                                  st["most"] + RESERVE, st["blocks"], case["dtype"], format="e2m1")
        st["cache"].bacon_cache_clear()
        st["cache"].bacon_cache_tables(st["batch"], None, RESERVE, st["free"])
        if op in ("step", "attend"):
            st["cache"].bacon_cache_store(st["batch"], list(st["k"]), list(st["v"]))
            del st["k"], st["v"]
    elif op in ("step", "attend"):
        # the cache as a program without the framework holds it: codes two to a byte, padded
        for name in ("k", "v"):
            y, e = _to_codes(_gather(st, name, st["most"] + case["new"])[0])
            st[name + "4"], st[name + "e"] = _pack(y), e.to(torch.int16)
            del st[name]
        st["rows"] = _rows(st)
        st["values"] = _pair_values()
    return st


# ---- the plain forms: positions

def _frequencies(case):
    """Turns a token of every pair in 64 bits, and what cos and sin are multiplied by."""
    r, base, s = case["rotary"], case["base"], case["factor"]
    if case["scaling"] == "ntk":
        base = base * s ** (r / (r - 2))
    f = torch.pow(torch.tensor(base, dtype=torch.float64, device="cuda"),
                  -torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r) / (2 * math.pi)
    if case["scaling"] == "linear":
        f = f / s
    if case["scaling"] == "yarn":
        keep = ((f * case["trained"] - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = f * keep + f / s * (1 - keep)
    return f, 0.1 * math.log(s) + 1.0 if case["scaling"] == "yarn" else 1.0


def _turn(st, x, weight):
    case, r = st["case"], st["case"]["rotary"]
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + NORM_EPS) * weight.float()
    p = st["positions"]
    if case["sections"]:
        row = torch.repeat_interleave(torch.arange(3, device="cuda"),
                                      torch.tensor(_ints(case["sections"]), device="cuda"), output_size=r // 2)
        p = p[row].t()
    else:
        p = p[:, None]
    t = p.double() * st["freq"]                                               # in turns, far positions among them
    t = (t - t.round()) * (2 * math.pi)
    cos, sin = (t.cos() * st["magnitude"]).float()[:, None], (t.sin() * st["magnitude"]).float()[:, None]
    if case["layout"] == "half":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        z = torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., r:]], -1)
    else:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        z = torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), y[..., r:]], -1)
    return z.to(x.dtype)


# ---- the plain forms: the prompt's attention

def _padded(x, cu, most):
    """Rows [T, H, d] as [B, H, most, d] in float32 (any rows of x behind a sequence's own)."""
    at = (cu[:-1, None] + torch.arange(most, device="cuda")).clamp_max(x.shape[0] - 1)
    return x[at].float().transpose(1, 2)


def _prompt_plain(st):
    case, cu, cuq = st["case"], st["cu_t"], st["cuq_t"]
    hq, hkv, d, W = case["hq"], case["hkv"], case["d"], case["window"]
    G, lens, nq = hq // hkv, st["len_t"], cuq[1:] - cuq[:-1]
    B, most, mostq = len(lens), max(_ints(case["lens"])), max(_ints(case["queries"]))
    q = (_padded(st["q"], cuq, mostq) / math.sqrt(d)).reshape(B * hkv, G * mostq, d)
    k = _padded(st["k"], cu, most).reshape(B * hkv, most, d)
    s = torch.bmm(q, k.transpose(1, 2)).view(B, hkv, G, mostq, most)
    del q, k
    end = (lens - nq)[:, None] + 1 + torch.arange(mostq, device="cuda")        # [B, mostq]
    unseen = torch.arange(most, device="cuda") >= end[..., None]
    s.masked_fill_(unseen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total))[..., 0].view(B, hq, mostq)
    out = torch.bmm(p.view(B * hkv, G * mostq, most), _padded(st["v"], cu, most).reshape(B * hkv, most, d))
    out = out.view(B, hkv, G, mostq, d) / total
    j = torch.arange(cuq[-1], device="cuda")
    b = torch.searchsorted(cuq[1:], j, right=True)
    i = j - cuq[b]
    rows = out.view(B, hq, mostq, d)[b, :, i].to(st["q"].dtype)
    w = nq[:, None] - W + torch.arange(W, device="cuda")                       # [B, W] queries of the window
    held = w >= 0
    window = lse.gather(2, w.clamp_min(0)[:, None].expand(B, hq, W))
    return {"out": rows, "lse": lse[b, :, i], "window": torch.where(held[:, None], window, 0.0)}


# ---- the plain forms: the cache

def _rows(st):
    W = st["case"]["window"]
    return torch.minimum(st["K"].long(), st["len_t"] - W) + W                  # [B], of every layer and head


def _two(e):
    """2^e as float32, for integers -126 <= e <= 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _to_codes(x):
    """Rows [.., d] of float32 as e2m1 values and the exponents [.., d / 32]: the
    smallest integers e with max |x| <= 6 2^e (6 is 0.75 times 2^3)."""
    y = x.unflatten(-1, (-1, GROUP))
    m, e = torch.frexp(y.abs().amax(-1))
    e = torch.where(m > 0, e - 3 + (m > 0.75).int(), E_LOW).clamp(E_LOW, E_HIGH)
    y = y / _two(e)[..., None]
    step = _two(torch.frexp(y)[1].sub(1).clamp_min(0) - 1)
    return (torch.round(y / step) * step).flatten(-2), e


def _pack(y):
    """Values as codes, two to a byte: the even dimension's in the low half."""
    a = y.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code = code + (torch.signbit(y).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _pair_values():
    """The two values of every byte [256, 2]."""
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    v = torch.cat([v, -v])
    i = torch.arange(256, device="cuda")
    return torch.stack([v[i & 15], v[i >> 4]], -1)


def _held(st, name):
    """The values that the plain cache holds, in float32."""
    y = st["values"][st[name + "4"].int()].flatten(-2)
    return (y.unflatten(-1, (-1, GROUP)) * _two(st[name + "e"])[..., None]).flatten(-2)


def _gather(st, name, cap):
    """The pairs' rows [L, B, Hkv, cap, d] as float32, zero beyond a pair's length."""
    x, W, rows = st[name], st["case"]["window"], _rows(st)
    L, H, B = x.shape[0], st["case"]["hkv"], len(rows)
    i = torch.arange(cap, device="cuda").expand(L, B, H, cap)
    kept = (rows - W)[None, :, None, None]
    at = i
    if "idx" in st:
        K = st["K"].long()
        h = torch.arange(H, device="cuda")
        start = (K.cumsum(0) - K)[:, None] * H + h * K[:, None]                # [B, H]
        flat = (start[None, :, :, None] + torch.minimum(i, (kept - 1).clamp_min(0))).reshape(L, -1)
        at = st["idx"].gather(1, flat.clamp_max(st["idx"].shape[1] - 1)).view(L, B, H, cap).long()
    at = torch.where(i < kept, at, i - kept + (st["len_t"] - W)[None, :, None, None])
    valid = i < rows[None, :, None, None]
    at = torch.where(valid, at + st["cu_t"][:-1][None, :, None, None], 0)
    l = torch.arange(L, device="cuda")[:, None, None, None]
    h = torch.arange(H, device="cuda")[None, None, :, None]
    return x[l, at, h].float() * valid[..., None]


def _store(st):
    got = {}
    for name in ("k", "v"):
        y, e = _to_codes(_gather(st, name, st["most"]))
        got[name] = (y.unflatten(-1, (-1, GROUP)) * _two(e)[..., None]).flatten(-2).to(_dtype(st["case"]))
    return got


def _count(st):
    n = st["case"]["new"]
    return torch.full_like(st["rows"], n) if st["counts"] is None else st["counts"].long()


def _append(st, name):
    """The new rows into the cache; the values of the last `new` rows of every pair."""
    n, rows, count = st["case"]["new"], st["rows"], _count(st)
    new = st[name + "_new"].float().transpose(1, 2)                            # [B, H, n, d]
    y, e = _to_codes(new)
    codes = _pack(y)
    B, H, _, half = codes.shape
    at = rows[:, None] + torch.arange(n, device="cuda")                        # [B, n]; rows of a token not taken stay
    fresh = (torch.arange(n, device="cuda") < count[:, None])[:, None, :, None]
    for held, x in ((st[name + "4"], codes), (st[name + "e"], e.to(torch.int16))):
        a = at[:, None, :, None].expand(B, H, n, x.shape[-1])
        held.scatter_(2, a, torch.where(fresh, x, held.gather(2, a)))
    pos = (rows + count - n)[:, None] + torch.arange(n, device="cuda")
    a = pos.clamp_min(0)[:, None, :, None]
    val = st["values"][st[name + "4"].gather(2, a.expand(B, H, n, half)).int()].flatten(-2)
    val = val.unflatten(-1, (-1, GROUP)) * _two(st[name + "e"].gather(2, a.expand(B, H, n, e.shape[-1])))[..., None]
    return (val.flatten(-2) * (pos >= 0)[:, None, :, None]).to(st[name + "_new"].dtype)[None]


def _attend(st, grown):
    q = st["q"]
    B, n, hq, d = q.shape
    H, G, count = st["case"]["hkv"], hq // st["case"]["hkv"], _count(st)
    total = st["rows"] + (count if grown else 0)
    cap = st["k4"].shape[2]
    k = _held(st, "k").view(B * H, cap, d)
    qq = q.float().view(B, n, H, G, d).transpose(1, 2).reshape(B * H, n * G, d) / math.sqrt(d)
    s = torch.bmm(qq, k.transpose(1, 2)).view(B, H, n, G, cap)
    del k
    j = torch.arange(n, device="cuda")
    end = total[:, None] - (count[:, None] - 1 - j)
    end = torch.where(j < count[:, None], end, 0)                              # [B, n]
    seen = torch.arange(cap, device="cuda") < end[:, None, :, None, None]
    s = torch.where(seen, s, -math.inf)
    top = s.amax(-1, keepdim=True).clamp_min(-1e30)
    p = torch.exp(s - top)
    del s
    total_p = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total_p))[..., 0]
    p = p / torch.where(total_p > 0, total_p, 1.0)
    out = torch.bmm(p.view(B * H, n * G, cap), _held(st, "v").view(B * H, cap, d))
    out = out.view(B, H, n, G, d).transpose(1, 2).reshape(B, n, hq, d).to(q.dtype)
    return out, lse.transpose(1, 2).reshape(B, n, hq)


def run(state):
    case, op = state["case"], state["op"]
    if own:
        bacon = state["bacon"]
        if op == "rotate":
            q, k = bacon.bacon_rotate(state["rotary"], state["positions"], state["q"], state["k"], state["q_norm"],
                                      state["k_norm"])
            return {"q": q, "k": k}
        if op == "prompt":
            window = torch.zeros(len(state["cu"]) - 1, case["hq"], case["window"], device="cuda")
            out, lse, window = bacon.bacon_prompt_attend(state["shape"], state["batch"], state["q"], state["k"],
                                                         state["v"], queries=state["cuq"], want_lse=True,
                                                         window_lse=window)
            return {"out": out, "lse": lse, "window": window}
        cache = state["cache"]
        if op == "store":
            cache.bacon_cache_store(state["batch"], state["k"], state["v"], state.get("idx"))
            k, v = cache.bacon_cache_load(state["most"])
            return {"k": k, "v": v}
        if op == "step":
            out, lse = cache.bacon_cache_step(0, state["q"], state["k_new"], state["v_new"], state["counts"],
                                              max_tokens=state["most"] + case["new"], want_lse=True)
            k, v = cache.bacon_cache_load(case["new"], first_token=-case["new"])
            cache.bacon_cache_advance(counts=state["back"])
            return {"out": out, "lse": lse, "k": k, "v": v}
        out, lse = cache.bacon_cache_attend(0, state["q"], state["counts"], max_tokens=state["most"], want_lse=True)
        return {"out": out, "lse": lse}
    if op == "rotate":
        return {"q": _turn(state, state["q"], state["q_norm"]), "k": _turn(state, state["k"], state["k_norm"])}
    if op == "prompt":
        return _prompt_plain(state)
    if op == "store":
        return _store(state)
    if op == "step":
        k, v = _append(state, "k"), _append(state, "v")
        out, lse = _attend(state, True)
        return {"out": out, "lse": lse, "k": k, "v": v}
    out, lse = _attend(state, False)
    return {"out": out, "lse": lse}


def work(case):
    """Each input read once and each output written once.  Rotation: queries and
    keys in and out, positions.  Prompt: queries, outputs, and every sequence's
    keys and values; products over the keys that each query sees.  Cache: the
    kept rows, their codes and scales (17 bytes for 32 values), and the rows read
    back; the codes of every row seen, queries, outputs, the new rows."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rotate":
        n = case["tokens"]
        return {"bytes": 2 * n * (hq + hkv) * d * es + 4 * n * (3 if case["sections"] else 1),
                "flops": 6 * n * (hq + hkv) * (case["rotary"] // 2)}
    lens = _ints(case["lens"])
    if case["op"] == "prompt":
        queries = _ints(case["queries"])
        nq, seen = sum(queries), sum(m * n - m * (m - 1) // 2 for m, n in zip(queries, lens))
        return {"bytes": 2 * nq * hq * d * es + 2 * sum(lens) * hkv * d * es
                + 4 * hq * (nq + sum(min(m, case["window"]) for m in queries)),
                "flops": 4 * seen * hq * d}
    L, W, n = case["layers"], case["window"], case["new"]
    pairs = L * len(lens) * hkv
    rows = L * hkv * sum(min(k, m - W) + W for k, m in zip(_ints(case["budgets"]), lens))
    held = 2 * rows * (d // 2 + d // GROUP)
    if case["op"] == "store":
        return {"bytes": 2 * rows * d * es + 2 * held + 2 * pairs * _most_rows(case) * d * es, "flops": 4 * rows * d}
    io = 2 * len(lens) * n * hq * d * es + held
    if case["op"] == "step":
        io += 2 * pairs * n * (2 * d * es + d // 2 + d // GROUP)
    return {"bytes": io, "flops": 4 * rows * n * (hq // hkv) * d}


# ---- the same results in 64 bits, from the definitions

def _exact_rotate(case, st):
    r, s, base = case["rotary"], case["factor"], case["base"]
    pairs, turned = r // 2, {}
    sections = _ints(case["sections"])
    angle = torch.zeros(case["tokens"], pairs, dtype=torch.float64, device="cuda")
    scale = 1.0
    for i in range(pairs):
        b = base * s ** (r / (r - 2)) if case["scaling"] == "ntk" else base
        omega = math.exp(-2.0 * i / r * math.log(b))
        if case["scaling"] == "linear":
            omega /= s
        elif case["scaling"] == "yarn":
            rotations = case["trained"] * omega / (2 * math.pi)
            gamma = 0.0 if rotations < 1 else 1.0 if rotations > 32 else (rotations - 1) / 31
            omega = (1 - gamma) * omega / s + gamma * omega
            scale = 0.1 * math.log(s) + 1.0
        p = st["positions"]
        if sections:
            p = p[0 if i < sections[0] else 1 if i < sections[0] + sections[1] else 2]
        angle[:, i] = p.double() * omega
    turn = torch.polar(torch.full_like(angle, scale), angle)[:, None]
    for name in ("q", "k"):
        x = st[name].double()
        w = st[name + "_norm"]
        if w is not None:
            x = x / (x.pow(2).sum(-1, keepdim=True) / case["d"] + NORM_EPS).sqrt() * w.double()
        i = torch.arange(pairs, device="cuda")
        re, im = (i, i + pairs) if case["layout"] == "half" else (2 * i, 2 * i + 1)
        z = torch.complex(x[..., re], x[..., im]) * turn
        y = x.clone()
        y[..., re], y[..., im] = z.real, z.imag
        turned[name] = y
    return turned


def _exact_prompt(case, st):
    hq, hkv, d, W = case["hq"], case["hkv"], case["d"], case["window"]
    queries, lens = _ints(case["queries"]), _ints(case["lens"])
    if hq * sum(m * n for m, n in zip(queries, lens)) > 8e9:
        return None
    nan = dict(dtype=torch.float64, device="cuda")
    out = torch.zeros(sum(queries), hq, d, **nan)
    lse = torch.zeros(sum(queries), hq, **nan)
    window = torch.zeros(len(lens), hq, W, **nan)
    for b, (m, n) in enumerate(zip(queries, lens)):
        k, v = (st[x][st["cu"][b]:st["cu"][b + 1]].double() for x in ("k", "v"))
        seen = torch.ones(m, n, dtype=torch.bool, device="cuda").tril(n - m)
        rows = slice(st["cuq"][b], st["cuq"][b + 1])
        for h in range(hq):
            s = st["q"][rows, h].double() @ k[:, h * hkv // hq].t().contiguous() / math.sqrt(d)
            s = s.masked_fill_(~seen, -math.inf)
            lse[rows, h] = torch.logsumexp(s, -1)
            out[rows, h] = torch.softmax(s, -1) @ v[:, h * hkv // hq]
        w = min(W, m)
        window[b, :, W - w:] = lse[rows][m - w:].t()
    return {"out": out, "lse": lse, "window": window}


def _exact_values(x):
    """Rows [n, d] in 64 bits as the cache holds them."""
    y = x.reshape(-1, GROUP)
    a = y.abs().amax(1)
    e = torch.ceil(torch.log2(a.clamp_min(2.0 ** -140) / 6.0))
    e = torch.where(6.0 * torch.pow(2.0, e - 1) >= a, e - 1, e)
    e = torch.where(6.0 * torch.pow(2.0, e) < a, e + 1, e).clamp(E_LOW, E_HIGH)
    scale = torch.pow(2.0, e)[:, None]
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
    z = y.abs() / scale
    lo = (torch.searchsorted(grid, z, right=True) - 1).clamp(0, 6)
    below, above = z - grid[lo], grid[lo + 1] - z
    up = (above < below) | ((above == below) & (lo % 2 == 1))
    return (torch.sign(y) * grid[lo + up.long()] * scale).view(x.shape)


def _exact_held(st, name, l, b, h):
    case = st["case"]
    W, n, K = case["window"], _ints(case["lens"])[b], _ints(case["budgets"])
    kept = min(K[b], n - W)
    if "idx" in st:
        start = sum(K[:b]) * case["hkv"] + h * K[b]
        at = st["idx"][l, start:start + kept].long()
    else:
        at = torch.arange(kept, device="cuda")
    at = torch.cat([at, torch.arange(n - W, n, device="cuda")]) + st["cu"][b]
    return _exact_values(st[name][l, at, h].double())


def exact(case, seed):
    st = _inputs(case, seed)
    if case["op"] == "rotate":
        return _exact_rotate(case, st)
    if case["op"] == "prompt":
        return _exact_prompt(case, st)
    L, hq, hkv, d, n = (case[x] for x in ("layers", "hq", "hkv", "d", "new"))
    B, G, most = len(_ints(case["lens"])), hq // hkv, _most_rows(case)
    wide = dict(dtype=torch.float64, device="cuda")
    if case["op"] == "store":
        if L * B * hkv > 4000 or L * B * hkv * most * d > 300_000_000:
            return None
        got = {x: torch.zeros(L, B, hkv, most, d, **wide) for x in ("k", "v")}
        for l in range(L):
            for b in range(B):
                for h in range(hkv):
                    for x in ("k", "v"):
                        rows = _exact_held(st, x, l, b, h)
                        got[x][l, b, h, :len(rows)] = rows
        return got
    out = torch.zeros(B, n, hq, d, **wide)
    lse = torch.full((B, n, hq), -math.inf, **wide)
    tails = {x: torch.zeros(1, B, hkv, n, d, **wide) for x in ("k", "v")}
    for b in range(B):
        c = n if st["counts"] is None else int(st["counts"][b])
        for h in range(hkv):
            kv = []
            for x in ("k", "v"):
                val = _exact_held(st, x, 0, b, h)
                if case["op"] == "step":
                    val = torch.cat([val, _exact_values(st[x + "_new"][b, :c, h].double())])
                    t = min(n, len(val))
                    tails[x][0, b, h, n - t:] = val[len(val) - t:]
                kv.append(val)
            k, v = kv
            for j in range(c):
                end = len(k) - (c - 1 - j)
                if end > 0:
                    s = st["q"][b, j, h * G:(h + 1) * G].double() @ k[:end].t().contiguous() / math.sqrt(d)
                    lse[b, j, h * G:(h + 1) * G] = torch.logsumexp(s, -1)
                    out[b, j, h * G:(h + 1) * G] = torch.softmax(s, -1) @ v[:end]
    if case["op"] == "step":
        return {"out": out, "lse": lse, "k": tails["k"], "v": tails["v"]}
    return {"out": out, "lse": lse}
