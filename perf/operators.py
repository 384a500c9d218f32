"""Performance cases of decoding over the kept rows in an 8-bit cache.

After the prompt's compression a serving program keeps the rows of every
(layer, sequence, KV head) in blocks of `bt` tokens, held in e4m3 with one
power-of-two scale for each block of K and of V, and decodes over them:

  tables   lengths, block tables and index offsets from the budgets, on the GPU
  store    the kept rows gathered and quantised into the blocks, and read back
           (a program that moves a compressed cache elsewhere)
  step     a decode step of one layer: the new tokens' rows appended, attention
           over the cache, the drafted tokens then rolled back (speculative
           decoding; the rows of the touched blocks are returned)
  attend   attention over the cache alone

`run` computes each in elementary torch operations, or with the framework's
calls where `own` is set.  A pair is a (layer, sequence, KV head).
"""
from __future__ import annotations

import math

import torch

own = False

E_LOW, E_HIGH, E4M3_MAX = -100, 120, 448.0
RESERVE = 64
LARGEST = 500_000_000        # values of K held by a drawn case, padded


def _case(name, op, layers, hq, hkv, d, window, bt, dtype, lens, budgets, new=1, spread=False,
          whole=False, counts=False, reserve=RESERVE):
    c = dict(op=op, layers=layers, hq=hq, hkv=hkv, d=d, window=window, bt=bt, dtype=dtype,
             lens=",".join(map(str, lens)), budgets=",".join(map(str, budgets)), new=new,
             spread=spread, whole=whole, counts=counts, reserve=reserve)
    return dict(name=name, **c) if name else c


def listed():
    ragged = (9631, 5167, 14011, 1291, 3083, 11117, 7411, 2049)
    full = tuple(n - 32 for n in ragged)
    many = tuple(900 + (i * 2377) % 7001 for i in range(64))
    mbud = tuple((64, 128, 512)[i % 3] for i in range(64))
    long32 = tuple(32768 - (i * 37) % 1021 for i in range(32))
    return [
        # the smallest prompt's cache: latency
        _case("tables-tiny", "tables", 2, 4, 4, 64, 8, 16, "fp32", (512,), (64,)),
        # a full serving batch with head-wise budgets that only the device knows
        _case("tables-adaptive-b64", "tables", 32, 32, 8, 128, 32, 16, "bf16", many, mbud, spread=True,
              reserve=1024),
        # the smallest prompt's kept rows
        _case("store-tiny-fp32", "store", 2, 4, 4, 64, 8, 16, "fp32", (512,), (64,)),
        # the headline prompt: 256 + 32 of 32K rows of every head and layer
        _case("store-video-32k", "store", 32, 32, 8, 128, 32, 64, "bf16", (32768,), (256,)),
        # a ragged batch kept whole (8 bits without compression)
        _case("store-ragged-whole", "store", 2, 32, 8, 128, 32, 32, "bf16", ragged, full, whole=True),
        # one token over the smallest cache
        _case("step-tiny-fp32", "step", 1, 4, 4, 64, 8, 16, "fp32", (512,), (64,), whole=True),
        # one token of one sequence over the headline's compressed cache
        _case("step-video-b1", "step", 1, 32, 8, 128, 32, 64, "bf16", (32768,), (256,), whole=True),
        # one token of 16 sequences, every query head with a KV head of its own
        _case("step-mha-b16", "step", 1, 32, 32, 128, 32, 16, "bf16", (2048,) * 16,
              tuple(64 + 37 * i for i in range(16)), whole=True),
        # up to four drafted tokens of 64 sequences over head-wise budgets
        _case("step-adaptive-b64", "step", 1, 28, 4, 128, 32, 32, "bf16", many, mbud, new=4, spread=True,
              whole=True, counts=True),
        # full precision, a small-head model, five tokens of four sequences
        _case("attend-fp32-n5", "attend", 1, 14, 2, 64, 16, 32, "fp32", (4099, 12289, 777, 8191),
              (4083, 12273, 761, 8175), new=5, whole=True),
        # a prompt of 128K tokens kept whole: one sequence over the whole GPU
        _case("attend-128k", "attend", 1, 32, 8, 128, 32, 64, "bf16", (131072,), (131040,), whole=True),
        # a batch of long prompts kept whole: bandwidth
        _case("attend-b32-32k", "attend", 1, 32, 8, 128, 32, 64, "bf16", long32,
              tuple(n - 32 for n in long32), whole=True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(("tables", "store", "step", "step", "attend", "attend", "attend"))
        hq, hkv = rng.choice(((4, 4), (32, 32), (28, 4), (32, 8), (14, 2), (32, 1), (64, 8)))
        d, bt = rng.choice((64, 128, 128)), rng.choice((16, 32, 64))
        window = rng.choice((1, 8, 16, 32))
        dtype = rng.choice(("bf16", "bf16", "bf16", "fp32"))
        batch = log_int(1, 64)
        layers = log_int(1, 32) if op in ("tables", "store") else 1
        new = rng.choice((1, 1, 1, 2, 3, 5, 8)) if op in ("step", "attend") else 1
        if hq // hkv * new > 64:
            continue
        top = {"tables": 32768, "store": 32768, "step": 8192, "attend": 131072}[op]
        mid = log_int(window + 1, top)
        lens = tuple(max(window, min(top, int(mid * math.exp(rng.uniform(-0.7, 0.7))))) for _ in range(batch))
        whole = op in ("step", "attend") or rng.random() < 0.3
        spread = op != "attend" and whole and rng.random() < 0.5 or op == "tables" and rng.random() < 0.5
        if whole and not spread:
            budgets = tuple(max(1, n - window) for n in lens)
        else:
            budgets = tuple(max(1, min(n - window, log_int(16, 1024))) for n in lens)
        rows = max(min((2 if spread else 1) * k, n - window) + window for k, n in zip(budgets, lens))
        if op != "tables" and layers * batch * hkv * rows * d > LARGEST:
            continue
        if layers * sum(lens) * hkv * d > LARGEST:
            if op != "tables" or layers * batch * hkv * (rows + RESERVE) * d > 4 * LARGEST:
                continue
        counts = new > 1 and batch > 1 and rng.random() < 0.5
        return _case(None, op, layers, hq, hkv, d, window, bt, dtype, lens, budgets, new, spread, whole, counts)


def _ints(s):
    return tuple(int(x) for x in s.split(","))


def _most_rows(case):
    """Upper bound of a pair's rows, as the program that sets the budgets knows it."""
    f = 2 if case["spread"] else 1
    return max(min(f * k, n - case["window"]) + case["window"]
               for k, n in zip(_ints(case["budgets"]), _ints(case["lens"])))


def _inputs(case, seed):
    """Unit-variance keys and values with a few strong channels and a strong
    first key (an attention sink), queries and new tokens' rows as views of one
    projection's output, budgets, kept positions and a shuffled free list."""
    L, hq, hkv, d, W = (case[x] for x in ("layers", "hq", "hkv", "d", "window"))
    lens, budgets, n = _ints(case["lens"]), _ints(case["budgets"]), case["new"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    B = len(lens)
    g = torch.Generator(device="cuda").manual_seed((seed * 1000003 + 29) & 0x7FFFFFFF)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    dev = dict(device="cuda")
    cu = torch.tensor([0] + list(lens)).cumsum(0).tolist()
    st = dict(op=case["op"], case=case, cu=cu)
    st["len_t"] = torch.tensor(lens, dtype=torch.int64, **dev)
    st["cu_t"] = torch.tensor(cu, dtype=torch.int64, **dev)
    K = torch.tensor(budgets, dtype=torch.int32, **dev)[None, :, None].expand(L, B, hkv)
    if case["spread"]:
        f = (0.6 * rnd(L, B, hkv)).exp().clamp(0.1, 2.0)
        K = (K * f).int().clamp_min(1)
    st["K"] = K.contiguous()
    rows = torch.minimum(K.long(), st["len_t"][None, :, None] - W) + W
    need = (rows + case["reserve"] + case["bt"] - 1) // case["bt"]
    st["blocks"] = int(need.sum()) + 3
    st["free"] = torch.randperm(st["blocks"], device="cuda", generator=g).int()
    if case["op"] != "tables":
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
        qkv = rnd(B, n, hq + 2 * hkv, d)
        qkv[..., :hq, :] *= 1.3
        qkv = qkv.to(dt)
        st["q"], st["k_new"], st["v_new"] = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
        st["counts"] = None
        if case["counts"]:
            st["counts"] = torch.randint(0, n + 1, (B,), dtype=torch.int32, device="cuda", generator=g)
        st["back"] = (torch.full((B,), -n, dtype=torch.int32, **dev) if st["counts"] is None
                      else -st["counts"])
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    bt = case["bt"]
    st["most"] = _most_rows(case)
    if own:
        from paper_2606_14782_amd import bacon
        lens, budgets = _ints(case["lens"]), _ints(case["budgets"])
        st["batch"] = bacon.BatchLayout(st["cu"], budgets)
        st["cache"] = bacon.Cache(case["layers"], case["hq"], case["hkv"], case["d"], case["window"], bt,
                                  len(lens), st["most"] + case["reserve"], st["blocks"], case["dtype"])
        st["cache"].bacon_cache_clear()
        st["budgets"] = st["K"] if case["spread"] else None
        if case["op"] != "tables":
            st["cache"].bacon_cache_tables(st["batch"], st["budgets"], case["reserve"], st["free"])
        if case["op"] in ("step", "attend"):
            st["cache"].bacon_cache_store(st["batch"], list(st["k"]), list(st["v"]))
            del st["k"], st["v"]
    elif case["op"] in ("step", "attend"):
        # the cache as a program without the framework holds it: padded, a row of blocks per pair
        blocks = st["most"] // bt + (bt + case["new"] - 2) // bt + 2
        for name in ("k", "v"):
            x = _gather(st, name, blocks * bt)[0]
            y, scale = _to_blocks(x.view(*x.shape[:2], blocks, bt, x.shape[-1]))
            st[name + "8"], st[name + "s"] = y.to(torch.float8_e4m3fn).view(torch.uint8), scale
            del x, y, st[name]
        st["rows"] = _rows(st)[0]
    return st


# ---- the plain forms

def _rows(st):
    W = st["case"]["window"]
    return torch.minimum(st["K"].long(), st["len_t"][None, :, None] - W) + W


def _starts(K):
    flat = K.reshape(K.shape[0], -1).long()
    return (flat.cumsum(1) - flat).view(K.shape)


def _two(e):
    """2^e as float32, for integers -126 <= e <= 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _exponent(a):
    """The smallest integer e, within bounds, with a <= 448 2^e (448 is 0.875 times 2^9)."""
    m, x = torch.frexp(a)
    return (x - 9 + (m > 0.875).int()).clamp(E_LOW, E_HIGH)


def _round8(x, scale):
    """x / scale rounded to the nearest e4m3 value, ties to even."""
    y = x / scale
    step = _two(torch.frexp(y)[1].sub(1).clamp_min(-6) - 3)
    return torch.round(y / step) * step


def _to_blocks(x):
    """Blocks [..., bt, d] of float32 rows as e4m3 values and scales [...]."""
    scale = _two(_exponent(x.abs().amax((-1, -2))))
    return _round8(x, scale[..., None, None]), scale


def _gather(st, name, cap):
    """The pairs' rows [L, B, Hkv, cap, d] as float32, zero beyond a pair's length."""
    x, W, rows = st[name], st["case"]["window"], _rows(st)
    L, B, H = rows.shape
    i = torch.arange(cap, device="cuda").expand(L, B, H, cap)
    kept = (rows - W)[..., None]
    at = i
    if "idx" in st:
        flat = (_starts(st["K"])[..., None] + torch.minimum(i, (kept - 1).clamp_min(0))).reshape(L, -1)
        at = st["idx"].gather(1, flat.clamp_max(st["idx"].shape[1] - 1)).view(L, B, H, cap).long()
    at = torch.where(i < kept, at, i - kept + (st["len_t"] - W)[None, :, None, None])
    valid = i < rows[..., None]
    at = torch.where(valid, at + st["cu_t"][:-1][None, :, None, None], 0)
    l = torch.arange(L, device="cuda")[:, None, None, None]
    h = torch.arange(H, device="cuda")[None, None, :, None]
    return x[l, at, h].float() * valid[..., None]


def _tables(st):
    case, K = st["case"], st["K"]
    bt, free = case["bt"], st["free"]
    most = (st["most"] + case["reserve"] + bt - 1) // bt
    rows = _rows(st)
    need = (rows + case["reserve"] + bt - 1) // bt
    first = need.reshape(-1).cumsum(0).view(need.shape) - need
    fits = (first + need <= free.numel()) & (need <= most)
    i = torch.arange(most, device="cuda")
    taken = (i < need[..., None]) & fits[..., None]
    table = torch.where(taken, free[(first[..., None] + i).clamp_max(free.numel() - 1)], -1)
    return {"lens": (rows * fits).int(), "starts": _starts(K).int(), "table": table, "used": need.sum().view(1)}


def _store(st):
    case = st["case"]
    bt = case["bt"]
    cap = (st["most"] + bt - 1) // bt * bt
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    got = {}
    for name in ("k", "v"):
        x = _gather(st, name, cap)
        y, scale = _to_blocks(x.view(*x.shape[:3], cap // bt, bt, x.shape[-1]))
        got[name] = (y * scale[..., None, None]).view(x.shape)[..., :st["most"], :].to(dt)
    return got


def _append(st, name):
    """The new rows into the blocks they touch; the last bt - 1 + n rows."""
    bt, n = st["case"]["bt"], st["case"]["new"]
    new, codes, scales, rows = st[name + "_new"], st[name + "8"], st[name + "s"], st["rows"]
    B, H, _, _, d = codes.shape
    nb = (bt + n - 2) // bt + 1
    blk = (rows // bt)[..., None] + torch.arange(nb, device="cuda")                   # [B, H, nb]
    pos = blk[..., None] * bt + torch.arange(bt, device="cuda")                       # [B, H, nb, bt]
    count = (torch.full_like(rows[:, 0], n) if st["counts"] is None else st["counts"].long())[:, None, None, None]
    j = pos - rows[..., None, None]
    fresh = ((j >= 0) & (j < count))[..., None]
    at = blk[..., None, None].expand(B, H, nb, bt, d)
    scale = scales.gather(2, blk)
    old = codes.gather(2, at).view(torch.float8_e4m3fn).float() * scale[..., None, None]
    b = torch.arange(B, device="cuda")[:, None, None, None]
    h = torch.arange(H, device="cuda")[None, :, None, None]
    x = torch.where(fresh, new[b, j.clamp(0, n - 1), h].float(), 0.0)
    need = _two(_exponent(x.abs().amax((-1, -2))))
    held = blk * bt < rows[..., None]
    touched = fresh.any(-2)[..., 0]
    scale = torch.where(touched, torch.where(held, torch.maximum(scale, need), need), scale)
    y = _round8(torch.where(fresh, x, old), scale[..., None, None])
    codes.scatter_(2, at, y.to(torch.float8_e4m3fn).view(torch.uint8))
    scales.scatter_(2, blk, scale)
    tail = bt - 1 + n
    pos = (rows[..., None] + count[..., 0] - tail) + torch.arange(tail, device="cuda")
    ok = pos >= 0
    pos = pos.clamp_min(0)
    val = codes.view(B, H, -1, d).gather(2, pos[..., None].expand(B, H, tail, d))
    val = val.view(torch.float8_e4m3fn).float() * scales.gather(2, pos // bt)[..., None]
    return (val * ok[..., None]).to(new.dtype)[None]


def _attend(st, grown):
    q = st["q"]
    B, n, hq, d = q.shape
    H, G = st["case"]["hkv"], hq // st["case"]["hkv"]
    count = torch.full_like(st["rows"][:, 0], n) if st["counts"] is None else st["counts"].long()
    total = st["rows"] + (count[:, None] if grown else 0)
    cap = st["k8"].shape[2] * st["k8"].shape[3]
    k = (st["k8"].view(torch.float8_e4m3fn).float() * st["ks"][..., None, None]).view(B * H, cap, d)
    qq = q.float().view(B, n, H, G, d).transpose(1, 2).reshape(B * H, n * G, d) / math.sqrt(d)
    s = torch.bmm(qq, k.transpose(1, 2)).view(B, H, n, G, cap)
    del k
    j = torch.arange(n, device="cuda")
    end = total[:, :, None] - (count[:, None, None] - 1 - j)
    end = torch.where(j < count[:, None, None], end, 0)                                # [B, H, n]
    seen = torch.arange(cap, device="cuda") < end[..., None, None]
    s = torch.where(seen, s, -math.inf)
    top = s.amax(-1, keepdim=True).clamp_min(-1e30)
    p = torch.exp(s - top)
    del s
    total_p = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total_p))[..., 0]
    p = p / torch.where(total_p > 0, total_p, 1.0)
    v = (st["v8"].view(torch.float8_e4m3fn).float() * st["vs"][..., None, None]).view(B * H, cap, d)
    out = torch.bmm(p.view(B * H, n * G, cap), v).view(B, H, n, G, d).transpose(1, 2)
    return out.reshape(B, n, hq, d).to(q.dtype), lse.transpose(1, 2).reshape(B, n, hq)


def run(state):
    case = state["case"]
    if own:
        cache = state["cache"]
        if case["op"] == "tables":
            used = cache.bacon_cache_tables(state["batch"], state["budgets"], case["reserve"], state["free"])
            return {"lens": cache.lens, "starts": cache.starts, "table": cache.table, "used": used}
        if case["op"] == "store":
            cache.bacon_cache_store(state["batch"], state["k"], state["v"], state.get("idx"))
            k, v = cache.bacon_cache_load(state["most"])
            return {"k": k, "v": v}
        if case["op"] == "step":
            out, lse = cache.bacon_cache_step(0, state["q"], state["k_new"], state["v_new"], state["counts"],
                                              max_tokens=state["most"] + case["new"], want_lse=True)
            tail = case["bt"] - 1 + case["new"]
            k, v = cache.bacon_cache_load(tail, first_token=-tail)
            cache.bacon_cache_advance(counts=state["back"])
            return {"out": out, "lse": lse, "k": k, "v": v}
        out, lse = cache.bacon_cache_attend(0, state["q"], state["counts"], max_tokens=state["most"], want_lse=True)
        return {"out": out, "lse": lse}
    if case["op"] == "tables":
        return _tables(state)
    if case["op"] == "store":
        return _store(state)
    if case["op"] == "step":
        k, v = _append(state, "k"), _append(state, "v")
        out, lse = _attend(state, True)
        return {"out": out, "lse": lse, "k": k, "v": v}
    out, lse = _attend(state, False)
    return {"out": out, "lse": lse}


def work(case):
    """Each input read once and each output written once: budgets, ids and
    tables; the kept rows, their codes, and the rows read back; the codes of
    every row seen, queries, outputs and the rows of the touched blocks."""
    L, hq, hkv, d, W, n, bt = (case[x] for x in ("layers", "hq", "hkv", "d", "window", "new", "bt"))
    es = 2 if case["dtype"] == "bf16" else 4
    lens, budgets = _ints(case["lens"]), _ints(case["budgets"])
    pairs = L * len(lens) * hkv
    most = _most_rows(case)
    rows = L * hkv * sum(min(k, m - W) + W for k, m in zip(budgets, lens))
    if case["op"] == "tables":
        blocks = (most + case["reserve"] + bt - 1) // bt
        return {"bytes": pairs * 4 * (blocks + 3) + 4 * (rows + pairs * case["reserve"]) // bt, "flops": 0}
    if case["op"] == "store":
        return {"bytes": 2 * d * (rows * (es + 2) + pairs * most * es), "flops": 4 * rows * d}
    io = 2 * len(lens) * n * hq * d * es + 2 * rows * d
    if case["op"] == "step":
        io += 2 * pairs * d * (n * (es + 1) + (bt - 1 + n) * es)
    return {"bytes": io, "flops": 4 * rows * n * (hq // hkv) * d}


# ---- the same results in 64 bits, from the definition

def _exact_block(x, least=None):
    """Values of a block of rows in 64 bits and its exponent (at least `least`)."""
    a = float(x.abs().max()) if x.numel() else 0.0
    e = E_LOW
    if a > 0:
        e = math.frexp(a)[1] - 10
        while E4M3_MAX * 2.0 ** e < a:
            e += 1
        e = min(max(e, E_LOW), E_HIGH)
    if least is not None:
        e = max(e, least)
    return _exact_values(x, 2.0 ** e), e


def _e4m3():
    v = [m * 2.0 ** -9 for m in range(8)]
    v += [(8 + m) * 2.0 ** (x - 10) for x in range(1, 16) for m in range(8)]
    return torch.tensor(v[:127], dtype=torch.float64, device="cuda")


def _exact_values(x, scale):
    table = _e4m3()
    y = x.abs() / scale
    lo = (torch.searchsorted(table, y, right=True) - 1).clamp(0, 125)
    below, above = y - table[lo], table[lo + 1] - y
    up = (above < below) | ((above == below) & (lo % 2 == 1))
    return torch.sign(x) * table[lo + up.long()] * scale


def _exact_rows(x, bt):
    """Rows [n, d] in 64 bits as the blocks hold them, and the blocks' exponents."""
    n, d = x.shape
    nb = (n + bt - 1) // bt
    pad = torch.zeros(nb * bt, d, dtype=torch.float64, device="cuda")
    pad[:n] = x
    a = pad.view(nb, -1).abs().amax(1)
    e = torch.ceil(torch.log2(a.clamp_min(1e-300) / E4M3_MAX))
    e = torch.where(E4M3_MAX * torch.pow(2.0, e - 1) >= a, e - 1, e)
    e = torch.where(E4M3_MAX * torch.pow(2.0, e) < a, e + 1, e).clamp(E_LOW, E_HIGH)
    scale = torch.tensor([2.0 ** int(t) for t in e.tolist()], dtype=torch.float64, device="cuda")
    return _exact_values(pad, scale.repeat_interleave(bt)[:, None])[:n], [int(t) for t in e.tolist()]


def _exact_held(st, name, l, b, h):
    case = st["case"]
    W, n = case["window"], _ints(case["lens"])[b]
    K = int(st["K"][l, b, h])
    kept = min(K, n - W)
    if "idx" in st:
        start = int(st["K"][l].reshape(-1)[:b * case["hkv"] + h].sum())
        at = st["idx"][l, start:start + kept].long()
    else:
        at = torch.arange(kept, device="cuda")
    at = torch.cat([at, torch.arange(n - W, n, device="cuda")]) + st["cu"][b]
    return st[name][l, at, h].double()


def exact(case, seed):
    st = _inputs(case, seed)
    if case["op"] == "tables":
        return None
    L, hq, hkv, d, bt, n = (case[x] for x in ("layers", "hq", "hkv", "d", "bt", "new"))
    B, G, most = len(_ints(case["lens"])), hq // hkv, _most_rows(case)
    if case["op"] == "store":
        if L * B * hkv > 2000:
            return None
        got = {x: torch.zeros(L, B, hkv, most, d, dtype=torch.float64, device="cuda") for x in ("k", "v")}
        for l in range(L):
            for b in range(B):
                for h in range(hkv):
                    for x in ("k", "v"):
                        rows = _exact_held(st, x, l, b, h)
                        got[x][l, b, h, :len(rows)] = _exact_rows(rows, bt)[0]
        return got
    out = torch.zeros(B, n, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((B, n, hq), -math.inf, dtype=torch.float64, device="cuda")
    tail = bt - 1 + n
    tails = {x: torch.zeros(1, B, hkv, tail, d, dtype=torch.float64, device="cuda") for x in ("k", "v")}
    for b in range(B):
        c = n if st["counts"] is None else int(st["counts"][b])
        for h in range(hkv):
            kv = []
            for x in ("k", "v"):
                val, es = _exact_rows(_exact_held(st, x, 0, b, h), bt)
                if case["op"] == "step":
                    new = st[x + "_new"][b, :c, h].double()
                    while len(new):
                        room = bt - len(val) % bt
                        part, new = new[:room], new[room:]
                        old = len(val) % bt
                        first = len(val) - old
                        _, e = _exact_block(part, es[first // bt] if old else None)
                        val = torch.cat([val[:first], _exact_values(torch.cat([val[first:], part]), 2.0 ** e)])
                    t = min(tail, len(val))
                    tails[x][0, b, h, tail - t:] = val[len(val) - t:]
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
