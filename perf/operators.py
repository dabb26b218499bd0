"""A request's way into the paged cache: the operators between a prompt and its first decode step, through the public binding.

Four operators of one model layer; a case names one by `op`:
  "slots"   block table and slot map of a step's new tokens, from the requests' lengths (hg_page_slots)
  "write"   the new tokens' K and V rows to their slots in the page pool, as bf16 or as E4M3 codes (hg_kv_write_paged)
  "prompt"  causal attention over whole prompts of different lengths, packed one after another (hg_prompt_attn)
  "chunk"   causal attention of every request's new tokens over its paged cache, single tokens among them (hg_chunk_attn_paged)
Fields: B requests; Hq, Hkv, D heads and head dimension; ctx_lo .. ctx_hi rows a request has in the cache before the step; new_lo .. new_hi
tokens it brings (`ones` of the requests bring a single one: they are decoding; some may bring none); page rows per page; cache "bf16" or "e4m3"; fused: Q, K and V
are views of one projection's output, so that rows lie further apart than they are long.
A case's lengths are evenly spread over their ranges, whatever the seed, which orders the requests.  Values are N(0, 1) rounded to bf16.
"""
import math

import torch

own = False

K_SCALE, V_SCALE = 0.0125, 0.011      # one step of the codes: 448 times this covers N(0, 1) with room


def _case(name, op, **more):
    c = dict(name=name, op=op, B=1, Hq=1, Hkv=1, D=128, ctx_lo=0, ctx_hi=0, new_lo=1, new_hi=1, ones=0, page=16, cache="bf16", fused=False)
    c.update(more)
    return c


def listed():
    return [
        # four requests of which some bring a short prompt: the smallest call, all latency
        _case("slots_small", "slots", B=4, ctx_lo=16, ctx_hi=500, new_lo=1, new_hi=64),
        # admission of 512 prompts at once: a slot for each of 130 thousand tokens
        _case("slots_admission", "slots", B=512, ctx_lo=0, ctx_hi=4096, new_lo=1, new_hi=512),
        # a decode step's rows of a small batch with grouped heads
        _case("write_step", "write", B=45, Hkv=2, D=128, ctx_lo=1, ctx_hi=150, new_lo=1, new_hi=1),
        # a 13b-class layer's prompts of up to 2K tokens into an 8-bit cache
        _case("write_prompts_codes", "write", B=16, Hkv=40, D=128, ctx_lo=0, ctx_hi=0, new_lo=1, new_hi=2048, cache="e4m3", fused=True),
        # four short prompts, a small model: launches and a chain of loads
        _case("prompt_tiny", "prompt", B=4, Hq=4, Hkv=4, D=64, new_lo=1, new_hi=64),
        # a ragged batch of short prompts with grouped heads
        _case("prompt_ragged", "prompt", B=45, Hq=16, Hkv=2, D=128, new_lo=1, new_hi=515),
        # prompts of up to 2K tokens in a 13b-class layer, read from the projection's output
        _case("prompt_2k", "prompt", B=16, Hq=40, Hkv=40, D=128, new_lo=1, new_hi=2048, fused=True),
        # one long document, 64 query heads on 8 KV heads
        _case("prompt_8k", "prompt", B=1, Hq=64, Hkv=8, D=128, new_lo=8192, new_hi=8192, fused=True),
        # single tokens of a small ragged batch: a decode step
        _case("chunk_tokens", "chunk", B=45, Hq=16, Hkv=2, D=128, ctx_lo=1, ctx_hi=515, ones=45),
        # prompts admitted into a running batch: most requests decode, eight bring up to 256 tokens
        _case("chunk_mixed", "chunk", B=64, Hq=32, Hkv=8, D=128, ctx_lo=1, ctx_hi=4096, new_lo=1, new_hi=256, ones=56),
        # a few drafted tokens behind long documents, 8-bit cache
        _case("chunk_long_codes", "chunk", B=3, Hq=64, Hkv=8, D=128, ctx_lo=16384, ctx_hi=65536, new_lo=1, new_hi=33, cache="e4m3", page=64),
        # the next 2K tokens of two long prompts over what is in the cache already
        _case("chunk_2k_over_16k", "chunk", B=2, Hq=64, Hkv=8, D=128, ctx_lo=8192, ctx_hi=16384, new_lo=1025, new_hi=2048),
    ]


# ---- what a case is made of --------------------------------------------------------------------------------------------------

def _spread(n, lo, hi):
    return [lo + (hi - lo) * i // max(n - 1, 1) if n > 1 else hi for i in range(n)]


def _requests(c):
    """[(rows in the cache, new tokens)] in a fixed order"""
    B, ones = c["B"], min(c["ones"], c["B"])
    ctx, new = _spread(B, c["ctx_lo"], c["ctx_hi"]), _spread(B - ones, c["new_lo"], c["new_hi"]) + [1] * ones
    step = next(s for s in range(max(1, int(B * 0.618)), 2 * B + 2) if math.gcd(s, B) == 1)      # long contexts with short and with long prompts
    return [(ctx[i * step % B], new[i]) for i in range(B)]


def _pages(n, ps):
    return -(-n // ps)


def _work_of(c):
    rq = _requests(c)
    T, B, kv, es = sum(n for _, n in rq), c["B"], c["Hkv"] * c["D"], 1 if c["cache"] == "e4m3" else 2
    if c["op"] == "slots":
        fresh = sum(_pages(x + n, c["page"]) - _pages(x, c["page"]) for x, n in rq)
        open_pages = sum(x % c["page"] != 0 for x, _ in rq)
        return {"bytes": 8.0 * B + 4 * open_pages + 8 * fresh + 4 * (B + 1) + 4 * T + 4 * B + 4, "flops": 0.0}
    if c["op"] == "write":
        return {"bytes": 2.0 * T * kv * (2 + es) + 4 * T, "flops": 0.0}
    io = T * c["Hq"] * (4.0 * c["D"] + 4)      # Q in, O and LSE out
    if c["op"] == "prompt":
        return {"bytes": io + 4.0 * T * kv, "flops": 4.0 * c["D"] * c["Hq"] * sum(n * (n + 1) / 2 for _, n in rq)}
    rows = sum(x + n for x, n in rq)
    return {"bytes": io + 2.0 * es * rows * kv + 4.0 * sum(_pages(x + n, c["page"]) for x, n in rq) + 8 * B,
            "flops": 4.0 * c["D"] * c["Hq"] * sum(n * x + n * (n + 1) / 2 for x, n in rq)}


def work(case):
    return _work_of(case)


def _plain_scores(c):
    """Elements of the plain form's padded score matrix."""
    longest = c["ctx_hi"] + (max(c["new_hi"], 1))
    return c["B"] * c["Hq"] * max(c["new_hi"], 1) * longest if c["op"] in ("prompt", "chunk") else 0


def draw(rng):
    heads = [(4, 4), (8, 1), (16, 2), (32, 8), (40, 40), (64, 8), (12, 4), (10, 2)]

    def log_int(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    cost = lambda c: _work_of(c)["bytes"] / 5e12 + _work_of(c)["flops"] / 1e15  # noqa: E731
    most = {op: max(cost(c) for c in listed() if c["op"] == op) for op in ("slots", "write", "prompt", "chunk")}
    while True:
        op = rng.choice(["slots", "write", "prompt", "prompt", "chunk", "chunk", "chunk"])
        Hq, Hkv = rng.choice(heads)
        new_hi = log_int(1, 8192) if op == "prompt" else log_int(1, 2048)
        ctx_hi = 0 if op == "prompt" else log_int(1, 65536)
        B = log_int(1, 512)
        c = dict(op=op, B=B, Hq=Hq, Hkv=Hkv, D=rng.choice([64, 128, 128]), ctx_lo=0 if op == "prompt" else log_int(1, ctx_hi), ctx_hi=ctx_hi,
                 new_lo=rng.randint(0, new_hi), new_hi=new_hi, ones=0 if op == "prompt" else rng.choice([0, B // 2, B - B // 8, B]),
                 page=rng.choice([16, 32, 64, 128]), cache=rng.choice(["bf16", "bf16", "e4m3"]) if op in ("write", "chunk") else "bf16",
                 fused=rng.random() < 0.5)
        rows = sum(x + n for x, n in _requests(c))
        if sum(n for _, n in _requests(c)) and cost(c) <= most[op] and _plain_scores(c) <= 5e9 and rows * Hkv * c["D"] < 1 << 29 and rows < 1 << 21:
            return c


# ---- inputs ------------------------------------------------------------------------------------------------------------------

def _values(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _qkv(c, g, T, queries=True):
    """Q, K, V rows of T tokens: tensors of their own, or views of one projection's output"""
    Hq, Hkv, D = c["Hq"] if queries else 0, c["Hkv"], c["D"]
    if not c["fused"]:
        return _values(g, T, Hq, D), _values(g, T, Hkv, D), _values(g, T, Hkv, D)
    x = _values(g, T, Hq + 2 * Hkv, D)
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]


def _pool(c, g, rows):
    if c["cache"] == "e4m3":
        return (_values(g, rows, c["Hkv"], c["D"]).float() / K_SCALE).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return _values(g, rows, c["Hkv"], c["D"])


def _inputs(c, seed):
    """Everything a case's operator reads, as tensors by name"""
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    cpu = torch.Generator().manual_seed(seed)
    rq = _requests(c)
    rq = [rq[i] for i in torch.randperm(len(rq), generator=cpu).tolist()]
    B, ps, ctx, new = c["B"], c["page"], [x for x, _ in rq], [n for _, n in rq]
    off = [0]
    for n in new:
        off.append(off[-1] + n)
    T, longest = off[-1], max(x + n for x, n in rq)
    s = {"ctx": _i32(ctx), "new": _i32(new), "q_off": _i32(off), "T": T, "max_new": max(new), "max_len": longest}
    if c["op"] == "prompt":
        s["Q"], s["K"], s["V"] = _qkv(c, g, T)
        return s
    # pages of the pool in a random order; every request's pages so far, and those of its new tokens from the list of free ones
    need = [(_pages(x, ps), _pages(x + n, ps)) for x, n in rq]
    stride, n_pages = max(w for _, w in need), sum(w for _, w in need) + 3
    order = torch.randperm(n_pages, generator=cpu).to(torch.int32)
    table = torch.full((B, stride), -1, dtype=torch.int32)
    at = 0
    for b, (have, _) in enumerate(need):
        table[b, :have] = order[at:at + have]
        at += have
    free = order[at:].clone()
    s["stride"] = stride
    if c["op"] == "slots":
        s["table"], s["free"] = table.cuda(), free.cuda()
        return s
    slots, at = torch.empty(T, dtype=torch.int32), 0
    for b, (have, want) in enumerate(need):
        table[b, have:want] = free[at:at + want - have]
        at += want - have
        j = torch.arange(ctx[b], ctx[b] + new[b])
        slots[off[b]:off[b + 1]] = table[b][j // ps] * ps + j % ps
    s["table"], s["slots"], s["len"] = table.cuda(), slots.cuda(), s["ctx"] + s["new"]
    s["Kp"], s["Vp"] = _pool(c, g, n_pages * ps), _pool(c, g, n_pages * ps)
    if c["op"] == "chunk":
        s["Q"] = _qkv(c, g, T)[0]
    else:
        _, s["K"], s["V"] = _qkv(c, g, T, queries=False)
        if T > 8:
            s["slots"][-1] = -1      # a batch padded to a fixed size: the last token is nobody's
    return s


def prepare(case, seed):
    """The step's tensors and the results', as a serving program keeps them"""
    s = _inputs(case, seed)
    s["case"] = case
    Hq, D, T = case["Hq"], case["D"], s["T"]
    if case["op"] in ("prompt", "chunk"):
        s["O"] = torch.empty(T, Hq, D, dtype=torch.bfloat16, device="cuda")
        s["LSE"] = torch.empty(T, Hq, dtype=torch.float32, device="cuda")
    if case["op"] == "slots":
        s["slots"] = torch.empty(T, dtype=torch.int32, device="cuda")
        s["offsets"], s["len"], s["used"] = torch.empty_like(s["q_off"]), torch.empty_like(s["ctx"]), torch.empty(1, dtype=torch.int32, device="cuda")
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------------

def _owner(off, T):
    """(request, position in it) of each of T packed tokens"""
    i = torch.arange(T, device=off.device)
    b = torch.searchsorted(off.long(), i, right=True) - 1
    return b, i - off.long()[b]


def _plain_slots(s, ps):
    x, n, free, stride = s["ctx"].long(), s["new"].long(), s["free"], s["stride"]
    have, want = (x + ps - 1) // ps, (x + n + ps - 1) // ps
    first = torch.cumsum(want - have, 0) - (want - have)
    col = torch.arange(stride, device=x.device)
    at = first[:, None] + col - have[:, None]
    mine = (col >= have[:, None]) & (col < want[:, None])
    table = torch.where(mine, free[at.clamp(0, free.numel() - 1)], s["table"])
    off = torch.cat([torch.zeros_like(n[:1]), torch.cumsum(n, 0)])
    b, t = _owner(off, s["T"])
    j = x[b] + t
    slots = table[b, j // ps].long() * ps + j % ps
    return {"page_table": table, "q_off": off.int(), "slots": slots.int(), "lengths": (x + n).int(), "used": (want - have).sum().reshape(1).int()}


def _plain_write(s, codes):
    slots, rows = s["slots"].long(), s["Kp"].shape[0]
    src = torch.full((rows + 1,), -1, dtype=torch.int64, device=slots.device)
    src[torch.where(slots >= 0, slots, rows)] = torch.arange(slots.numel(), device=slots.device)
    src = src[:rows]
    out = []
    for pool, new, scale in ((s["Kp"], s["K"], K_SCALE), (s["Vp"], s["V"], V_SCALE)):
        if codes:
            new = (new.float() / torch.tensor(scale, dtype=torch.float32, device=new.device)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        out.append(torch.where((src >= 0)[:, None, None], new[src.clamp(min=0)], pool))
    return {"K": out[0].view(torch.float8_e4m3fn) if codes else out[0], "V": out[1].view(torch.float8_e4m3fn) if codes else out[1]}


def _plain_attention(c, Q, q_off, k, v, lens, new, max_new):
    """Q: packed tokens; k, v: fp32 [B, longest, Hkv, D]; token t of a request's n sees rows [0, len - (n - 1 - t))"""
    B, L, Hkv, D = k.shape
    T, Hq, G = Q.shape[0], Q.shape[1], Q.shape[1] // Hkv
    pos = torch.arange(max_new, device=Q.device)
    at = (q_off[:-1].long()[:, None] + pos).clamp(max=T - 1)
    q = Q.float()[at].view(B, max_new, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B * Hkv, G * max_new, D)
    kt = k.permute(0, 2, 3, 1).reshape(B * Hkv, D, L)
    sc = torch.matmul(q, kt).view(B, Hkv, G, max_new, L).mul_(1.0 / math.sqrt(D))
    seen = (lens.long() - new.long())[:, None] + pos + 1
    sc.masked_fill_((torch.arange(L, device=Q.device) >= seen[:, :, None])[:, None, None], -math.inf)
    m = sc.amax(-1, keepdim=True)
    p = sc.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B * Hkv, G * max_new, L), v.permute(0, 2, 1, 3).reshape(B * Hkv, L, D)).view(B, Hkv, G, max_new, D) / l
    lse = (m + l.log())[..., 0]
    b, t = _owner(q_off, T)
    return {"O": o.permute(0, 3, 1, 2, 4).reshape(B, max_new, Hq, D)[b, t].to(torch.bfloat16), "LSE": lse.permute(0, 3, 1, 2).reshape(B, max_new, Hq)[b, t]}


def _cache_rows(s, c, dtype):
    """K and V of every request's rows, padded to the longest: [B, longest, Hkv, D]"""
    j = torch.arange(s["max_len"], device="cuda")
    rows = s["table"][:, j // c["page"]].long().clamp(min=0) * c["page"] + j % c["page"]
    here = (j < s["len"][:, None])[:, :, None, None]
    out = []
    for pool, scale in ((s["Kp"], K_SCALE), (s["Vp"], V_SCALE)):
        x = pool[rows]
        x = x.view(torch.float8_e4m3fn).to(dtype) * scale if c["cache"] == "e4m3" else x.to(dtype)
        out.append(torch.where(here, x, torch.zeros((), dtype=dtype, device="cuda")))
    return out


def _prompt_rows(s, dtype):
    at = (s["q_off"][:-1].long()[:, None] + torch.arange(s["max_new"], device="cuda")).clamp(max=s["T"] - 1)
    return s["K"][at].to(dtype), s["V"][at].to(dtype)


def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    if c["op"] == "slots":
        return _plain_slots(s, c["page"])
    if c["op"] == "write":
        return _plain_write(s, c["cache"] == "e4m3")
    if c["op"] == "prompt":
        k, v = _prompt_rows(s, torch.float32)
        return _plain_attention(c, s["Q"], s["q_off"], k, v, s["new"], s["new"], s["max_new"])
    k, v = _cache_rows(s, c, torch.float32)
    return _plain_attention(c, s["Q"], s["q_off"], k, v, s["len"], s["new"], s["max_new"])


_handle = None


def _library():
    """The binding and the program's one context, with a workspace that fits every case"""
    global _handle
    from paper_2402_05099_amd import binding as hb
    if _handle is None:
        _handle = hb.Context(0, 512 << 20)
    return hb, _handle


def _run_own(s, c):
    hb, h = _library()
    if "Kp" in s and "kv" not in s:
        s["kv"] = hb.PagedKV(K=s["Kp"], V=s["Vp"], page_table=s["table"], page_size=c["page"],
                             kv_format=hb.HG_KV_E4M3 if c["cache"] == "e4m3" else hb.HG_KV_BF16, k_scale=K_SCALE, v_scale=V_SCALE)
    if c["op"] == "slots":
        hb.hg_page_slots(h, s["ctx"], s["new"], s["free"], c["page"], s["table"], s["offsets"], s["slots"], s["len"], s["used"])
        return {"page_table": s["table"], "q_off": s["offsets"], "slots": s["slots"], "lengths": s["len"], "used": s["used"]}
    if c["op"] == "write":
        hb.hg_kv_write_paged(h, s["K"], s["V"], s["slots"], s["kv"])
        return {n: s[p].view(torch.float8_e4m3fn) if c["cache"] == "e4m3" else s[p] for n, p in (("K", "Kp"), ("V", "Vp"))}
    if c["op"] == "prompt":
        hb.hg_prompt_attn(h, s["Q"], s["K"], s["V"], s["q_off"], s["max_new"], s["O"], s["LSE"])
    else:
        hb.hg_chunk_attn_paged(h, s["Q"], s["q_off"], s["kv"], s["len"], s["max_new"], s["max_len"], s["O"], s["LSE"])
    return {"O": s["O"], "LSE": s["LSE"]}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------

def _e4m3_values():
    """The 256 values of the format: sign, 4 exponent bits with bias 7, 3 mantissa bits, NaN where all of them are set"""
    v = []
    for code in range(256):
        e, f = (code >> 3) & 15, code & 7
        x = math.nan if (code & 127) == 127 else f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
        v.append(-x if code & 128 else x)
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def exact(case, seed):
    s, c = _inputs(case, seed), case
    if c["op"] == "slots":
        return None
    if c["op"] == "write":
        val, here, out = _e4m3_values(), s["slots"] >= 0, {}
        for name, scale in (("K", K_SCALE), ("V", V_SCALE)):
            pool = val[s[name + "p"].long()] if c["cache"] == "e4m3" else s[name + "p"].double()
            new = s[name].double()
            if c["cache"] == "e4m3":
                new = (new / scale).clamp(-448, 448)
            pool[s["slots"][here].long()] = new[here]
            out[name] = pool
        return out
    T, Hq, Hkv, D = s["T"], c["Hq"], c["Hkv"], c["D"]
    O = torch.empty(T, Hq, D, dtype=torch.float64, device="cuda")
    LSE = torch.empty(T, Hq, dtype=torch.float64, device="cuda")
    off = s["q_off"].tolist()
    val = _e4m3_values()
    for b in range(c["B"]):
        n = off[b + 1] - off[b]
        if n == 0:
            continue
        rows = int(s["len"][b]) if c["op"] == "chunk" else n
        if c["op"] == "chunk":
            at = torch.cat([torch.arange(c["page"], device="cuda") + p * c["page"] for p in s["table"][b].tolist() if p >= 0])[:rows]
        for kvh in range(Hkv):
            if c["op"] == "prompt":
                k, v = (s[x][off[b]:off[b + 1], kvh].double() for x in ("K", "V"))
            elif c["cache"] == "e4m3":
                k, v = val[s["Kp"][at, kvh].long()] * K_SCALE, val[s["Vp"][at, kvh].long()] * V_SCALE
            else:
                k, v = s["Kp"][at, kvh].double(), s["Vp"][at, kvh].double()
            for h in range(kvh * (Hq // Hkv), (kvh + 1) * (Hq // Hkv)):
                z = s["Q"][off[b]:off[b + 1], h].double() @ k.T.contiguous() / math.sqrt(D)
                late = torch.arange(rows, device="cuda")[None, :] - torch.arange(n, device="cuda")[:, None] > rows - n
                w = z.masked_fill(late, -math.inf)
                LSE[off[b]:off[b + 1], h] = torch.logsumexp(w, 1)
                O[off[b]:off[b + 1], h] = torch.softmax(w, 1) @ v
    return {"O": O, "LSE": LSE}
