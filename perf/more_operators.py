"""Timing cases of the 8-bit paged cache: rows quantised as they are written to their pages, rows read back, and attention
over the 8-bit pages.  The cache holds e4m3 values and a scale for every block of tokens and head; a written block's scale is
the smallest power of two that keeps the block within the type's 448.  ``run`` computes the operators in plain torch operations,
or, with ``own`` set, through this package's entry points."""
import math

import torch

own = False

DEV = "cuda"
F8 = torch.float8_e4m3fn
TOP = 448.0


# ------------------------------------------------------------------------------------------------ cases
def _attn(name, B, Hq, Hkv, D, n_q, lo, hi, ps=16, block=16, dtype="bf16", causal=True, window=0, sinks=0, ragged=False):
    c = dict(op="attn", B=B, Hq=Hq, Hkv=Hkv, D=D, n_q=n_q, lo=lo, hi=hi, ps=ps, block=block, dtype=dtype, causal=causal,
             window=window, sinks=sinks, ragged=ragged)
    return dict(c, name=name) if name else c


def _write(name, B, Hkv, D, old_lo, old_hi, n_lo, n_hi, ps=16, block=16, dtype="bf16"):
    c = dict(op="write", B=B, Hkv=Hkv, D=D, old_lo=old_lo, old_hi=old_hi, n_lo=n_lo, n_hi=n_hi, ps=ps, block=block, dtype=dtype)
    return dict(c, name=name) if name else c


def _read(name, B, Hkv, D, lo, hi, ps=16, block=16, dtype="bf16", dense=False, skip=0):
    c = dict(op="read", B=B, Hkv=Hkv, D=D, lo=lo, hi=hi, ps=ps, block=block, dtype=dtype, dense=dense, skip=skip)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one request, one new token, a short prompt: latency
        _attn("attn8-1x1-short", 1, 32, 32, 128, 1, 769, 769),
        # a batch of grouped-query requests of uneven lengths, one new token each
        _attn("attn8-gqa-16x1", 16, 28, 4, 128, 1, 300, 4096, ps=32, block=32),
        # a full batch of long multi-head caches, one new token each: the largest
        _attn("attn8-mha-32x1-long", 32, 32, 32, 128, 1, 4096, 4160),
        # a decoding block of 32 positions that see each other and the whole prefix
        _attn("attn8-block32-8", 8, 32, 32, 128, 32, 1024, 2080, ps=64, block=64, causal=False),
        # the same of a grouped-query model: 224 query rows share each key
        _attn("attn8-gqa-block32-16", 16, 28, 4, 128, 32, 1500, 4128, ps=64, block=64, causal=False),
        # one very long grouped-query document, a scale for every token: split over the length and joined
        _attn("attn8-gqa-1x1-131k", 1, 28, 4, 128, 1, 131072, 131072, ps=64, block=1),
        # fp32 queries, a few drafted tokens per request, sliding window with first tokens that stay visible
        _attn("attn8-f32-window", 24, 16, 8, 64, 4, 50, 9000, ps=16, block=8, dtype="f32", window=1000, sinks=4, ragged=True),
        # one decode step: every request adds a row to a block that holds others already
        _write("write8-decode-64", 64, 4, 128, 30, 4000, 1, 1),
        # prompts of uneven lengths
        _write("write8-prefill-32", 32, 32, 128, 0, 0, 17, 2048, ps=64, block=64),
        # fp32, a block of 32 rows per request, part of it in a block begun before
        _write("write8-f32-block32", 101, 8, 64, 0, 3000, 32, 32, ps=24, block=12, dtype="f32"),
        # prefixes of a batch laid out densely for the attention over a dense prefix cache
        _read("read8-dense-16", 16, 32, 128, 500, 2048, ps=64, block=64, dense=True),
        # the rows of a few requests behind a shared beginning, packed, in fp32
        _read("read8-f32-packed", 5, 8, 64, 30, 3001, ps=24, block=8, dtype="f32", skip=17),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "write", "read"])
    ps, block = rng.choice([(1, 1), (8, 8), (8, 2), (16, 16), (16, 4), (24, 12), (24, 3), (32, 1), (64, 64), (64, 16), (128, 128)])
    f32 = rng.random() < 0.3
    dtype = "f32" if f32 else "bf16"
    if op == "attn":
        D = rng.choice([64, 128])
        Hkv, G = rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 2, 4, 7, 8])
        n_q = rng.choice([1, 1, 1, 2, 3, 5, 8, 16, 32, 33])
        B = _log(rng, 1, 64)
        room = int(min(0.7e9 / (B * Hkv * D * 2), 8e9 / (4 * B * Hkv * G * n_q * D)))
        hi = max(n_q, min(131072, _log(rng, 16, 131072), room))
        lo = rng.choice([0, n_q, hi // 3, hi])
        win = rng.choice([0, 0, 1, 77, 1024])
        return _attn(None, B, Hkv * G, Hkv, D, n_q, min(lo, hi), hi, ps, block, dtype, causal=rng.random() < 0.6, window=win,
                     sinks=rng.choice([0, 4, 17]) if win else 0, ragged=rng.random() < 0.4)
    D, Hkv = rng.choice([64, 96, 128, 256]), rng.choice([1, 2, 4, 8, 32])
    rows = max(1, min(_log(rng, 1, 32768), int(9e7 / (Hkv * D))))
    if op == "write":
        B = _log(rng, 1, max(2, min(512, rows)))
        n_hi = max(1, rows // B)
        old_hi = _log(rng, 1, max(2, min(4096, int(2e8 / (B * Hkv * D)))))
        return _write(None, B, Hkv, D, rng.choice([0, old_hi]), old_hi, rng.choice([1, n_hi]), n_hi, ps, block, dtype)
    B = _log(rng, 1, max(2, min(64, rows)))
    hi = max(1, rows // B)
    return _read(None, B, Hkv, D, rng.choice([0, hi]), hi, ps, block, dtype, dense=rng.random() < 0.5, skip=rng.choice([0, 0, hi // 2]))


# ------------------------------------------------------------------------------------------------ inputs
def _spread(n, lo, hi):
    """n lengths over [lo, hi], the last one hi, the same for every seed (their order is the seed's)."""
    return [hi if i == n - 1 else lo + int((hi - lo) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _shuffled(values, rng):
    return torch.tensor(values)[torch.randperm(len(values), generator=rng)].to(torch.int32)


def _starts(counts):
    return torch.cat([torch.zeros(1, dtype=torch.int64), torch.as_tensor(counts).long().cumsum(0)]).to(torch.int32)


def _queries(c):
    return [max(1, c["n_q"] // 2) if c["ragged"] and b % 3 == 1 else c["n_q"] for b in range(c["B"])]


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _cache(gen, n_pages, c):
    """Pages of one cache as a serving process finds them: rows of uneven size, quantised block by block."""
    ps, T, H, D = c["ps"], c["block"], c["Hkv"], c["D"]
    codes = torch.empty(n_pages, H, ps, D, dtype=F8, device=DEV)
    scales = torch.empty(n_pages, H, ps // T, dtype=torch.float32, device=DEV)
    step = max(1, (1 << 27) // (H * ps * D))
    for p in range(0, n_pages, step):
        x = torch.empty(min(step, n_pages - p), H, ps // T, T, D, dtype=torch.float32, device=DEV).normal_(generator=gen)
        x *= torch.empty(x.shape[:4], dtype=torch.float32, device=DEV).normal_(0.0, 0.4, generator=gen).exp_()[..., None]
        s = _power(_exponent(x.abs().amax((-1, -2)), 0.875, 9))
        scales[p:p + step] = s
        codes[p:p + step] = (x / s[..., None, None]).view(-1, H, ps, D).to(F8)
    return codes, scales


def prepare(case, seed):
    c = dict(case)
    host = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device=DEV).manual_seed(seed + 1)

    def normal(*shape):
        return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=gen)

    s, op, B, D, ps, dt = {"case": c}, c["op"], c["B"], c["D"], c["ps"], _dtype(c)
    if op == "write":
        old, new = _shuffled(_spread(B, c["old_lo"], c["old_hi"]), host), _shuffled(_spread(B, c["n_lo"], c["n_hi"]), host)
        lens = old + new
        per = -(-(c["old_hi"] + c["n_hi"]) // ps)
    else:
        lens = _shuffled(_spread(B, c["lo"], c["hi"]), host)
        per = max(1, -(-c["hi"] // ps))
    n_pages = B * per + 3
    s["table"] = torch.randperm(n_pages, generator=host)[:B * per].view(B, per).to(torch.int32).to(DEV)
    s["kv_len"] = lens.to(DEV)
    s["k_cache"], s["k_scale"] = _cache(gen, n_pages, c)
    s["v_cache"], s["v_scale"] = _cache(gen, n_pages, c)
    if op == "attn":
        starts = _starts(_queries(c))
        N = int(starts[-1])
        # heads look at more or less sharply chosen places
        sharp = torch.linspace(0.5, 3.0, c["Hq"], device=DEV).view(1, -1, 1)
        s["q"] = (normal(N, c["Hq"], D) * sharp).to(dt)
        s["row_start"] = starts.to(DEV)
        s["scale"] = 1.0 / math.sqrt(D)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(N, c["Hq"], dtype=torch.float32, device=DEV)
    elif op == "write":
        starts = _starts(new)
        N = int(starts[-1])
        # rows of uneven size, some larger than what their blocks hold already
        size = torch.empty(N, c["Hkv"], 1, dtype=torch.float32, device=DEV).normal_(0.0, 0.8, generator=gen).exp_()
        s["k"], s["v"] = (normal(N, c["Hkv"], D) * size).to(dt), (normal(N, c["Hkv"], D) * size).to(dt)
        s["row_start"], s["max_q"], s["max_len"] = starts.to(DEV), c["n_hi"], c["old_hi"] + c["n_hi"]
    else:
        first = torch.minimum(lens, torch.full_like(lens, c["skip"]))
        s["first"] = first.to(DEV)
        if c["dense"]:
            s["k_out"] = torch.zeros(B, c["hi"], c["Hkv"], D, dtype=dt, device=DEV)
        else:
            starts = _starts(lens - first)
            s["out_start"] = starts.to(DEV)
            s["k_out"] = torch.zeros(max(1, int(starts[-1])), c["Hkv"], D, dtype=dt, device=DEV)
        s["v_out"] = torch.zeros_like(s["k_out"])
    if own:
        # the fixed arguments of a decoding loop's call, checked once; the loop then only launches it
        import paper_2601_17917_b200 as ds
        cache = (s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"], s["kv_len"])
        if op == "attn":
            s["plan"] = ds.PagedAttn8Plan(s["q"], *cache, s["scale"], row_start=s["row_start"], max_q=c["n_q"], max_len=c["hi"],
                                          causal=c["causal"], window=c["window"], sinks=c["sinks"], out=s["out"], lse=s["lse"])
        elif op == "write":
            s["plan"] = ds.Kv8WritePlan(s["k"], s["v"], *cache, row_start=s["row_start"], max_q=s["max_q"], max_len=s["max_len"])
        else:
            s["plan"] = ds.Kv8ReadPlan(*cache, s["k_out"], s["v_out"], out_start=s.get("out_start"), first=s["first"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _values(codes, scales):
    """Pages [.., ps, D] of codes with scales [.., ps / block] -> fp32."""
    x = codes.float()
    return (x.unflatten(-2, (scales.shape[-1], -1)) * scales[..., None, None]).flatten(-3, -2)


def _plain_attn(s):
    c, q = s["case"], s["q"]
    B, Hq, Hkv, D, n_q = c["B"], c["Hq"], c["Hkv"], c["D"], c["n_q"]
    L = s["table"].shape[1] * c["ps"]
    first, count = s["row_start"][:-1].long(), s["row_start"].long().diff()
    i = torch.arange(n_q, device=q.device)
    real = i < count[:, None]
    rows = torch.where(real, first[:, None] + i, 0)
    qp = q[rows].float().view(B, n_q, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    t = s["table"].long()
    k = _values(s["k_cache"][t], s["k_scale"][t]).permute(0, 2, 1, 3, 4).reshape(B, Hkv, L, D)
    z = (qp @ k.transpose(-1, -2)).mul_(s["scale"]).view(B, Hkv, Hq // Hkv, n_q, L)
    del k
    lens = s["kv_len"].long()
    end = (lens - count + 1)[:, None] + i if c["causal"] else lens[:, None].expand(B, n_q)
    at = torch.arange(L, device=q.device)
    see = at < end[..., None]
    if c["window"]:
        see &= (at < c["sinks"]) | (at >= (end - c["window"])[..., None])
    z.masked_fill_(~see[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = _values(s["v_cache"][t], s["v_scale"][t]).permute(0, 2, 1, 3, 4).reshape(B, Hkv, L, D)
    o = (p.view(B, Hkv, -1, L) @ v).view(B, Hkv, Hq // Hkv, n_q, D) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log()).squeeze(-1)
    s["out"][rows[real]] = o.permute(0, 3, 1, 2, 4).reshape(B, n_q, Hq, D)[real].to(q.dtype)
    s["lse"][rows[real]] = lse.permute(0, 3, 1, 2).reshape(B, n_q, Hq)[real]
    return {"out": s["out"], "lse": s["lse"]}


def _exponent(x, top_mantissa, shift):
    """The smallest e, not below -126, with x <= 2 top_mantissa 2^(shift - 1) 2^e; x >= 0 and finite."""
    m, e = torch.frexp(x)
    e = torch.where(m <= top_mantissa, e - shift, e - shift + 1)
    return torch.where(x == 0, -126, e).clamp(min=-126)


def _power(e):
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _plain_write_one(s, x, codes, scales):
    """Quantises the rows x [N, Hkv, D] into their blocks; rows that the first of a sequence's blocks holds already are
    rescaled with it."""
    c = s["case"]
    ps, T = c["ps"], c["block"]
    x = x.float()
    starts, lens, t = s["row_start"].long(), s["kv_len"].long(), s["table"].long()
    r = torch.arange(x.shape[0], device=x.device)
    b = torch.searchsorted(starts[1:].contiguous(), r, right=True)
    old = lens - starts.diff()
    pos = old[b] + r - starts[b]
    page, off = t[b, pos // ps], pos % ps
    blocks = ps // T
    flat = scales.transpose(1, 2).reshape(-1, c["Hkv"])                          # [pages * blocks, Hkv]
    which = page * blocks + off // T
    need = torch.zeros_like(flat).scatter_reduce_(0, which[:, None].expand(-1, c["Hkv"]), x.abs().amax(-1), "amax")
    e = _exponent(need, 0.875, 9)
    # rows held before, in the block that a sequence's first new row falls into
    j = torch.arange(T, device=x.device)
    before = old[:, None] // T * T + j
    held = (before < old[:, None]) & (starts.diff() > 0)[:, None]
    before = before[held]
    hb = torch.arange(len(old), device=x.device)[:, None].expand(-1, T)[held]
    hpage, hoff = t[hb, before // ps], before % ps
    hwhich = hpage * blocks + hoff // T
    e[hwhich] = torch.maximum(e[hwhich], _exponent(flat[hwhich], 0.5, 1))
    new = _power(e)
    codes[hpage, :, hoff] = (codes[hpage, :, hoff].float() * (flat[hwhich] / new[hwhich])[..., None]).to(F8)
    codes[page, :, off] = (x / new[which][..., None]).to(F8)
    scales[page, :, off // T] = new[which]


def _plain_write(s):
    _plain_write_one(s, s["k"], s["k_cache"], s["k_scale"])
    _plain_write_one(s, s["v"], s["v_cache"], s["v_scale"])
    return _write_outputs(s)


def _write_outputs(s):
    # the 8-bit values as they are and the scales that they are multiplied by
    return {n: s[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")}


def _plain_read(s):
    c, t, lens, first = s["case"], s["table"].long(), s["kv_len"].long(), s["first"].long()
    ps, T = c["ps"], c["block"]
    if c["dense"]:
        i = torch.arange(c["hi"], device=t.device)
        there = i < (lens - first)[:, None]
        b = torch.arange(c["B"], device=t.device)[:, None].expand_as(there)[there]
        pos = (first[:, None] + i)[there]
        to = there
    else:
        r = torch.arange(int(s["k_out"].shape[0]), device=t.device)
        starts = s["out_start"].long()
        b = torch.searchsorted(starts[1:].contiguous(), r, right=True)
        to = b < c["B"]
        b = b.clamp(max=c["B"] - 1)
        pos = torch.where(to, first[b] + r - starts[b], 0)
        b, pos = b[to], pos[to]
    page, off = t[b, pos // ps], pos % ps
    s["k_out"][to] = (s["k_cache"][page, :, off].float() * s["k_scale"][page, :, off // T][..., None]).to(s["k_out"].dtype)
    s["v_out"][to] = (s["v_cache"][page, :, off].float() * s["v_scale"][page, :, off // T][..., None]).to(s["v_out"].dtype)
    return {"k": s["k_out"], "v": s["v_out"]}


def run(state):
    op = state["case"]["op"]
    if own:
        state["plan"].launch()
        if op == "attn":
            return {"out": state["out"], "lse": state["lse"]}
        return _write_outputs(state) if op == "write" else {"k": state["k_out"], "v": state["v_out"]}
    return {"attn": _plain_attn, "write": _plain_write, "read": _plain_read}[op](state)


# ------------------------------------------------------------------------------------------------ work and 64 bits
def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    row = c["Hkv"] * (c["D"] + 4.0 / c["block"])      # bytes of a row of one 8-bit cache
    if c["op"] == "attn":
        queries, lens = sorted(_queries(c)), _spread(c["B"], c["lo"], c["hi"])
        # how many rows a sequence of which length has is the seed's; the mean of them is not
        n = sum(queries) / len(queries)
        keys = products = 0.0
        for length in lens:
            for i in range(int(n)):
                end = max(0, length - int(n) + 1 + i if c["causal"] else length)
                products += min(end, min(c["sinks"], end) + c["window"]) if c["window"] else end
            first = max(0, length - int(n) + 1) if c["causal"] else length
            keys += length if not c["window"] else min(length, c["sinks"] + c["window"] + length - first)
        products *= n / int(n)
        io = 2 * sum(queries) * c["Hq"] * c["D"] * es + 4 * sum(queries) * c["Hq"]
        return {"bytes": 2 * keys * row + io + 4 * keys / c["ps"], "flops": 4 * products * c["Hq"] * c["D"]}
    if c["op"] == "write":
        rows = sum(_spread(c["B"], c["n_lo"], c["n_hi"]))
    else:
        rows = sum(n - min(n, c["skip"]) for n in _spread(c["B"], c["lo"], c["hi"]))
    rows = max(1, rows)
    return {"bytes": 2 * rows * (row + c["Hkv"] * c["D"] * es) + 4 * rows / c["ps"], "flops": 4 * rows * c["Hkv"] * c["D"]}


def _exact_attn(s):
    c = s["case"]
    G, ps, T = c["Hq"] // c["Hkv"], c["ps"], c["block"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    starts, lens = s["row_start"].tolist(), s["kv_len"].tolist()
    for b, length in enumerate(lens):
        if length == 0:
            continue
        pages = s["table"][b, :-(-length // ps)].long()
        for h in range(c["Hkv"]):
            k, v = (x[pages, h].double().reshape(-1, c["D"])[:length] * f[pages, h].double().reshape(-1).repeat_interleave(T)[:length, None]
                    for x, f in ((s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"])))
            for i, r in enumerate(range(starts[b], starts[b + 1])):
                end = length - (starts[b + 1] - starts[b]) + 1 + i if c["causal"] else length
                if end <= 0:
                    continue
                if c["window"] and end - c["window"] > c["sinks"]:
                    see = [slice(0, c["sinks"]), slice(end - c["window"], end)]
                else:
                    see = [slice(0, end)]
                kk, vv = torch.cat([k[a] for a in see]), torch.cat([v[a] for a in see])
                z = torch.einsum("gd,td->gt", s["q"][r, h * G:(h + 1) * G].double(), kk) * s["scale"]
                l = torch.logsumexp(z, 1)
                out[r, h * G:(h + 1) * G] = (z - l[:, None]).exp() @ vv
                lse[r, h * G:(h + 1) * G] = l
    return {"out": out, "lse": lse}


def _nearest_e4m3(x):
    """Nearest multiple of the spacing at |x| (3 bits behind the first, never finer than 2^-9), ties to even."""
    size = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    unit = torch.exp2(size - 3)
    return torch.round(x / unit) * unit


def _exact_write(s):
    c = s["case"]
    ps, T, H, D = c["ps"], c["block"], c["Hkv"], c["D"]
    got = {n: s[n].double() for n in ("k_cache", "v_cache", "k_scale", "v_scale")}
    starts, lens = s["row_start"].tolist(), s["kv_len"].tolist()
    for b, length in enumerate(lens):
        n = starts[b + 1] - starts[b]
        if n == 0:
            continue
        lo = (length - n) // T * T                       # the sequence's rows from the first block that is written on
        hi = -(-length // T) * T
        pos = torch.arange(lo, hi, device=DEV)
        page, off = s["table"][b, pos // ps].long(), pos % ps
        fresh, gone = pos >= length - n, pos >= length
        for name in ("k", "v"):
            codes, scales = got[name + "_cache"], got[name + "_scale"]
            held = codes[page, :, off]                    # [rows, H, D]
            f = scales[page, :, off // T]                 # [rows, H]
            x = held * f[..., None]
            mine = fresh & ~gone
            x[mine] = s[name][starts[b]:starts[b + 1]].double()
            peak = torch.where(mine[:, None], x.abs().amax(-1), 0.0).view(-1, T, H).amax(1)
            # a scale that rows in the block have already is never lowered
            least = torch.where((~fresh)[:, None], f, 0.0).view(-1, T, H).amax(1)
            up = torch.exp2(torch.round(torch.log2((peak / TOP).clamp(min=2.0 ** -126))))      # one of the two next to it
            by = torch.where(up * TOP < peak, 2 * up, torch.where(up * TOP >= 2 * peak, up / 2, up).clamp(min=2.0 ** -126))
            by = torch.maximum(by, least)
            rows = by.repeat_interleave(T, 0)
            codes[page, :, off] = torch.where(gone[:, None, None], held, _nearest_e4m3(x / rows[..., None]))
            scales[page[::T], :, off[::T] // T] = by
    return got


def _exact_read(s):
    c = s["case"]
    ps, T = c["ps"], c["block"]
    k, v = torch.zeros(s["k_out"].shape, dtype=torch.float64, device=DEV), torch.zeros(s["k_out"].shape, dtype=torch.float64, device=DEV)
    lens, first, at = s["kv_len"].tolist(), s["first"].tolist(), 0
    for b, length in enumerate(lens):
        pos = torch.arange(first[b], length, device=DEV)
        page, off = s["table"][b, pos // ps].long(), pos % ps
        for out, codes, scales in ((k, s["k_cache"], s["k_scale"]), (v, s["v_cache"], s["v_scale"])):
            rows = codes[page, :, off].double() * scales[page, :, off // T].double()[..., None]
            if c["dense"]:
                out[b, :len(pos)] = rows
            else:
                out[at:at + len(pos)] = rows
        at += len(pos)
    return {"k": k, "v": v}


def exact(case, seed):
    if case["op"] == "attn" and case["B"] * case["Hkv"] * case["n_q"] > 20000:
        return None
    s = prepare(case, seed)
    return {"attn": _exact_attn, "write": _exact_write, "read": _exact_read}[case["op"]](s)
