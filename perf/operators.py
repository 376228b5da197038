"""Timing cases of the paged-cache operators: page bookkeeping, per-head norm + rotary position + cache write,
and attention over the paged cache.  ``run`` computes them in plain torch operations, or, with ``own`` set, through
this package's entry points."""
import math

import torch

own = False

DEV = "cuda"
THETA = 1000000.0


# ------------------------------------------------------------------------------------------------ cases
def _attn(name, B, Hq, Hkv, D, n_q, lo, hi, ps=16, dtype="bf16", causal=True, window=0, sinks=0, ragged=False):
    c = dict(op="attn", B=B, Hq=Hq, Hkv=Hkv, D=D, n_q=n_q, lo=lo, hi=hi, ps=ps, dtype=dtype, causal=causal,
             window=window, sinks=sinks, ragged=ragged)
    return dict(c, name=name) if name else c


def _rope(name, N, Hq, Hkv, D, rot, ps=16, dtype="bf16", interleaved=False, norm=True, factor=1.0, pos=32768):
    c = dict(op="rope", N=N, Hq=Hq, Hkv=Hkv, D=D, rot=rot, ps=ps, dtype=dtype, interleaved=interleaved, norm=norm,
             factor=factor, pos=pos)
    return dict(c, name=name) if name else c


def _pages(name, B, ps, old_lo, old_hi, new_lo, new_hi, done_every):
    c = dict(op="pages", B=B, ps=ps, old_lo=old_lo, old_hi=old_hi, new_lo=new_lo, new_hi=new_hi, done_every=done_every)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one request, one new token, a short prompt: latency
        _attn("attn-1x1-short", 1, 32, 32, 128, 1, 769, 769),
        # a batch of grouped-query requests of uneven lengths, one new token each
        _attn("attn-gqa-16x1", 16, 28, 4, 128, 1, 300, 4096, ps=32),
        # a full batch of long multi-head caches, one new token each: the largest
        _attn("attn-mha-32x1-long", 32, 32, 32, 128, 1, 4096, 4160),
        # a decoding block of 32 positions that see each other and the whole prefix
        _attn("attn-block32-8", 8, 32, 32, 128, 32, 1024, 2080, ps=64, causal=False),
        # one very long grouped-query document: split over the length and joined
        _attn("attn-gqa-1x1-131k", 1, 28, 4, 128, 1, 131072, 131072, ps=64),
        # fp32, a few drafted tokens per request, sliding window with first tokens that stay visible
        _attn("attn-f32-window", 24, 16, 8, 64, 4, 50, 9000, dtype="f32", window=1000, sinks=4, ragged=True),
        # one decode step of a batch: a few dozen rows, latency
        _rope("rope-decode-32", 32, 32, 32, 128, 128),
        # a long prompt of a grouped-query model with frequencies scaled for long contexts
        _rope("rope-prefill-gqa", 16384, 28, 4, 128, 128, ps=64, factor=4.0, pos=131072),
        # fp32, interleaved pairs, part of the head rotated, an odd number of rows
        _rope("rope-f32-partial", 4099, 16, 8, 64, 32, dtype="f32", interleaved=True),
        # every request of a decode step grows by one row
        _pages("pages-decode-256", 256, 16, 30, 4000, 1, 1, 0),
        # continuous batching: an eighth of the requests have finished, the others add a prompt piece
        _pages("pages-prefill-64", 64, 16, 0, 3000, 1, 4000, 8),
        # a large server's step: some requests finish, the others add a block of 32
        _pages("pages-block-2048", 2048, 32, 0, 2000, 32, 32, 16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "rope", "pages"])
    if op == "attn":
        f32 = rng.random() < 0.3
        D = rng.choice([32, 64, 128, 256] if f32 else [64, 128])
        Hkv, G = rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 2, 4, 7, 8])
        n_q = rng.choice([1, 1, 1, 2, 3, 5, 8, 16, 32, 33])
        B = _log(rng, 1, 64)
        room = int(min(0.8e9 / (B * Hkv * D * (8 if f32 else 4)), 8e9 / (4 * B * Hkv * G * n_q * D)))
        hi = max(n_q, min(131072, _log(rng, 16, 131072), room))
        lo = rng.choice([0, n_q, hi // 3, hi])
        win = rng.choice([0, 0, 1, 77, 1024])
        return _attn(None, B, Hkv * G, Hkv, D, n_q, min(lo, hi), hi, ps=rng.choice([1, 8, 16, 24, 64, 128]),
                     dtype="f32" if f32 else "bf16", causal=rng.random() < 0.6, window=win,
                     sinks=rng.choice([0, 4, 17]) if win else 0, ragged=rng.random() < 0.4)
    if op == "rope":
        f32 = rng.random() < 0.3
        D = rng.choice([64, 96, 128, 256])
        rot = rng.choice([D, D, 32, 64])
        Hkv, G = rng.choice([1, 4, 8, 32]), rng.choice([1, 4, 7])
        N = max(1, min(_log(rng, 1, 16384), int(7e7 / (Hkv * (G + 2) * D))))
        return _rope(None, N, Hkv * G, Hkv, D, rot, ps=rng.choice([1, 16, 24, 64]), dtype="f32" if f32 else "bf16",
                     interleaved=rng.random() < 0.5, norm=rng.random() < 0.7, factor=rng.choice([1.0, 1.0, 4.0, 16.0]),
                     pos=rng.choice([64, 4096, 131072, 1000000]))
    B = _log(rng, 1, 2048)
    new_hi = _log(rng, 1, max(2, min(8192, 130000 // B)))
    old_hi = _log(rng, 1, min(8192, max(2, 4000000 // B)))
    return _pages(None, B, rng.choice([1, 8, 16, 24, 64, 128]), rng.choice([0, old_hi]), old_hi,
                  rng.choice([0, new_hi]), new_hi, rng.choice([0, 2, 5, 16]))


# ------------------------------------------------------------------------------------------------ inputs
def _spread(n, lo, hi):
    """n lengths over [lo, hi], the last one hi, the same for every seed (their order is the seed's)."""
    return [hi if i == n - 1 else lo + int((hi - lo) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _shuffled(values, rng):
    return torch.tensor(values)[torch.randperm(len(values), generator=rng)].to(torch.int32)


def _queries(c):
    return [max(1, c["n_q"] // 2) if c["ragged"] and b % 3 == 1 else c["n_q"] for b in range(c["B"])]


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    c = dict(case)
    host = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device=DEV).manual_seed(seed + 1)

    def normal(*shape):
        return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=gen)

    s = {"case": c}
    if c["op"] == "attn":
        B, D, ps, dt = c["B"], c["D"], c["ps"], _dtype(c)
        lens = _shuffled(_spread(B, c["lo"], c["hi"]), host)
        per = -(-c["hi"] // ps)
        n_pages = B * per + 3
        starts = torch.tensor([0] + _queries(c)).cumsum(0).to(torch.int32)
        N = int(starts[-1])
        # heads look at more or less sharply chosen places
        sharp = torch.linspace(0.5, 3.0, c["Hq"], device=DEV).view(1, -1, 1)
        s["q"] = (normal(N, c["Hq"], D) * sharp).to(dt)
        s["k_cache"] = normal(n_pages, c["Hkv"], ps, D).to(dt)
        s["v_cache"] = normal(n_pages, c["Hkv"], ps, D).to(dt)
        s["table"] = torch.randperm(n_pages, generator=host)[:B * per].view(B, per).to(torch.int32).to(DEV)
        s["kv_len"], s["row_start"] = lens.to(DEV), starts.to(DEV)
        s["scale"] = 1.0 / math.sqrt(D)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(N, c["Hq"], dtype=torch.float32, device=DEV)
    elif c["op"] == "rope":
        N, Hq, Hkv, D, ps, dt = c["N"], c["Hq"], c["Hkv"], c["D"], c["ps"], _dtype(c)
        qkv = normal(N, Hq + 2 * Hkv, D).mul_(2.0).to(dt)    # the fused projection's output
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["q_weight"] = (1.0 + 0.1 * normal(D)).to(dt) if c["norm"] else None
        s["k_weight"] = (1.0 + 0.1 * normal(D)).to(dt) if c["norm"] else None
        s["positions"] = torch.randint(0, c["pos"], (N,), generator=host, dtype=torch.int32).to(DEV)
        n_pages = -(-N // ps) + 2
        s["slots"] = torch.randperm(n_pages * ps, generator=host)[:N].to(DEV)
        s["k_cache"] = torch.zeros(n_pages, Hkv, ps, D, dtype=dt, device=DEV)
        s["v_cache"] = torch.zeros_like(s["k_cache"])
        s["q_out"] = torch.empty(N, Hq, D, dtype=dt, device=DEV)
    else:
        B, ps = c["B"], c["ps"]
        old = _shuffled(_spread(B, c["old_lo"], c["old_hi"]), host)
        new = _shuffled(_spread(B, c["new_lo"], c["new_hi"]), host)
        done = torch.zeros(B, dtype=torch.uint8)
        if c["done_every"]:
            done[torch.randperm(B, generator=host)[:B // c["done_every"]]] = 1
            new[done.bool()] = 0
        width = -(-(c["old_hi"] + c["new_hi"]) // ps)
        n_pages = B * width
        perm = torch.randperm(n_pages, generator=host).to(torch.int32)
        held = (old + ps - 1) // ps
        table = torch.zeros(B, width, dtype=torch.int32)
        used = int(held.sum())
        table[torch.arange(width)[None, :] < held[:, None]] = perm[:used]
        free = torch.zeros(n_pages, dtype=torch.int32)
        free[:n_pages - used] = perm[used:]
        s["kv_len"], s["n_new"], s["done"] = old.to(DEV), new.to(DEV), done.to(DEV)
        s["table"], s["free_list"] = table.to(DEV), free.to(DEV)
        s["free_cnt"] = torch.tensor([n_pages - used], dtype=torch.int32, device=DEV)
        s["max_rows"] = B * c["new_hi"]
        s["kv_len_out"], s["free_cnt_out"] = torch.empty_like(s["kv_len"]), torch.empty_like(s["free_cnt"])
        s["row_start"] = torch.empty(B + 1, dtype=torch.int32, device=DEV)
        s["positions"] = torch.empty(max(1, s["max_rows"]), dtype=torch.int32, device=DEV)[:s["max_rows"]]
        s["slots"] = torch.empty(max(1, s["max_rows"]), dtype=torch.int64, device=DEV)[:s["max_rows"]]
    if own:
        # the fixed arguments of a decoding loop's call, checked once; the loop then only launches it
        import paper_2601_17917_b200 as ds
        if c["op"] == "attn":
            s["plan"] = ds.PagedAttnPlan(s["q"], s["k_cache"], s["v_cache"], s["table"], s["kv_len"], s["scale"],
                                         row_start=s["row_start"], max_q=c["n_q"], max_len=c["hi"], causal=c["causal"],
                                         window=c["window"], sinks=c["sinks"], out=s["out"], lse=s["lse"])
        elif c["op"] == "rope":
            rope = ds.RopeTable(c["rot"], THETA, interleaved=c["interleaved"], **_scaling(c))
            s["plan"] = ds.QkNormRopePlan(s["q"], s["k"], s["v"], s["positions"], rope, q_weight=s["q_weight"],
                                          k_weight=s["k_weight"], eps=1e-6, q_out=s["q_out"], k_cache=s["k_cache"],
                                          v_cache=s["v_cache"], slot_map=s["slots"])
        else:
            s["plan"] = ds.PageUpdatePlan(s["kv_len"], s["n_new"], s["table"], s["free_list"], s["free_cnt"], c["ps"],
                                          done=s["done"], kv_len_out=s["kv_len_out"], free_cnt_out=s["free_cnt_out"],
                                          row_start=s["row_start"], positions=s["positions"], slot_map=s["slots"])
    return s


def _scaling(c):
    """By-parts scaling (YaRN) for a context `factor` times the 32768 positions of the original one."""
    if c["factor"] == 1.0:
        return {}
    return dict(scaling="yarn", factor=c["factor"], orig_len=32768, beta_fast=32.0, beta_slow=1.0)


# ------------------------------------------------------------------------------------------------ plain forms
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
    k = s["k_cache"][t].permute(0, 2, 1, 3, 4).reshape(B, Hkv, L, D).float()
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
    v = s["v_cache"][t].permute(0, 2, 1, 3, 4).reshape(B, Hkv, L, D).float()
    o = (p.view(B, Hkv, -1, L) @ v).view(B, Hkv, Hq // Hkv, n_q, D) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log()).squeeze(-1)
    s["out"][rows[real]] = o.permute(0, 3, 1, 2, 4).reshape(B, n_q, Hq, D)[real].to(q.dtype)
    s["lse"][rows[real]] = lse.permute(0, 3, 1, 2).reshape(B, n_q, Hq)[real]
    return {"out": s["out"], "lse": s["lse"]}


def _frequencies(c, device):
    """Angles per position of the rotated pairs (64 bits), and the factor on the rotated values."""
    d = torch.arange(0, c["rot"], 2, dtype=torch.float64, device=device)
    f = THETA ** (-d / c["rot"])
    sc = _scaling(c)
    if not sc:
        return f, 1.0
    turns = [c["rot"] * math.log(sc["orig_len"] / (b * 2 * math.pi)) / (2 * math.log(THETA))
             for b in (sc["beta_fast"], sc["beta_slow"])]
    lo, hi = max(math.floor(turns[0]), 0), min(math.ceil(turns[1]), c["rot"] - 1)
    ramp = ((d / 2 - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
    return f * (1.0 - ramp) + f / sc["factor"] * ramp, 0.1 * math.log(sc["factor"]) + 1.0


def _plain_norm_rope(s, x, w):
    c, R = s["case"], s["case"]["rot"]
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w.float()
    f, m = _frequencies(c, x.device)
    a = s["positions"].double()[:, None] * f
    cos, sin = (a.cos() * m).float()[:, None], (a.sin() * m).float()[:, None]
    r = y[..., :R]
    lo, hi = (r[..., 0::2], r[..., 1::2]) if c["interleaved"] else (r[..., :R // 2], r[..., R // 2:])
    pair = (lo * cos - hi * sin, hi * cos + lo * sin)
    r = torch.stack(pair, -1).flatten(-2) if c["interleaved"] else torch.cat(pair, -1)
    return torch.cat([r, y[..., R:]], -1).to(x.dtype)


def _plain_rope(s):
    s["q_out"].copy_(_plain_norm_rope(s, s["q"], s["q_weight"]))
    page, off = s["slots"] // s["case"]["ps"], s["slots"] % s["case"]["ps"]
    s["k_cache"][page, :, off] = _plain_norm_rope(s, s["k"], s["k_weight"])
    s["v_cache"][page, :, off] = s["v"]
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_pages(s):
    ps, width, n_rows = s["case"]["ps"], s["table"].shape[1], s["max_rows"]
    length, new, done = s["kv_len"].long(), s["n_new"].long(), s["done"].bool()
    table, stack, free = s["table"], s["free_list"], s["free_cnt"].long()
    col = torch.arange(width, device=table.device)
    back = torch.where(done, (length + ps - 1) // ps, 0)
    at = free + back.cumsum(0)[:, None] - back[:, None] + col
    mine = col < back[:, None]
    stack[at[mine]] = table[mine]
    free = free + back.sum()
    old = torch.where(done, 0, length)
    have = (old + ps - 1) // ps
    need = (old + new + ps - 1) // ps - have
    upto = need.cumsum(0)
    given = ((need == 0) | (upto <= free)) & (new.cumsum(0) <= n_rows) & (have + need <= width)
    need, new = torch.where(given, need, 0), torch.where(given, new, 0)
    nth = col - have[:, None]
    mine = (nth >= 0) & (nth < need[:, None])
    table[mine] = stack[(free - 1 - (upto - need)[:, None] - nth)[mine]]
    s["kv_len_out"].copy_(old + new)
    s["free_cnt_out"].copy_(free - need.sum())
    s["row_start"][0] = 0
    s["row_start"][1:] = new.cumsum(0)
    r = torch.arange(n_rows, device=table.device)
    b = torch.searchsorted(new.cumsum(0), r, right=True)
    used = b < len(new)
    b = b.clamp(max=len(new) - 1)
    pos = torch.where(used, old[b] + r - s["row_start"][b], 0)
    slot = table[b, pos // ps].long() * ps + pos % ps
    s["positions"].copy_(pos)
    s["slots"].copy_(torch.where(used, slot, -1))
    return _page_outputs(s)


def _page_outputs(s):
    return {n: s[n] for n in ("kv_len_out", "free_cnt_out", "row_start", "positions", "slots", "table", "free_list")}


def run(state):
    op = state["case"]["op"]
    if own:
        state["plan"].launch()
        if op == "attn":
            return {"out": state["out"], "lse": state["lse"]}
        if op == "rope":
            return {"q": state["q_out"], "k_cache": state["k_cache"], "v_cache": state["v_cache"]}
        return _page_outputs(state)
    return {"attn": _plain_attn, "rope": _plain_rope, "pages": _plain_pages}[op](state)


# ------------------------------------------------------------------------------------------------ work and 64 bits
def work(case):
    c = case
    if c["op"] == "attn":
        es, queries, lens = (4 if c["dtype"] == "f32" else 2), sorted(_queries(c)), _spread(c["B"], c["lo"], c["hi"])
        # how many rows a sequence of which length has is the seed's; the mean of them is not
        n = sum(queries) / len(queries)
        keys = products = 0.0
        for length in lens:
            for i in range(int(n)):
                end = length - int(n) + 1 + i if c["causal"] else length
                end = max(0, end)
                products += min(end, min(c["sinks"], end) + c["window"]) if c["window"] else end
            first = max(0, length - int(n) + 1) if c["causal"] else length
            keys += length if not c["window"] else min(length, c["sinks"] + c["window"] + length - first)
        products *= n / int(n)
        io = 2 * sum(queries) * c["Hq"] * c["D"] * es + 4 * sum(queries) * c["Hq"]
        return {"bytes": 2 * keys * c["Hkv"] * c["D"] * es + io + 4 * keys / c["ps"],
                "flops": 4 * products * c["Hq"] * c["D"]}
    if c["op"] == "rope":
        es = 4 if c["dtype"] == "f32" else 2
        x = c["N"] * (c["Hq"] + 2 * c["Hkv"]) * c["D"]
        return {"bytes": 2 * x * es + 12 * c["N"], "flops": x * (8 if c["norm"] else 4)}
    old, new = _spread(c["B"], c["old_lo"], c["old_hi"]), _spread(c["B"], c["new_lo"], c["new_hi"])
    done = c["B"] // c["done_every"] if c["done_every"] else 0
    live = 1.0 - done / c["B"]
    moved = sum(old) / c["ps"] * (done / c["B"]) + sum(new) * live / c["ps"]
    return {"bytes": 21 * c["B"] + 8 * moved + 12 * c["B"] * c["new_hi"], "flops": 12 * c["B"] + 4 * c["B"] * c["new_hi"]}


def _exact_attn(s):
    c = s["case"]
    G, ps = c["Hq"] // c["Hkv"], c["ps"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    starts, lens = s["row_start"].tolist(), s["kv_len"].tolist()
    for b, length in enumerate(lens):
        if length == 0:
            continue
        pages = s["table"][b, :-(-length // ps)].long()
        for h in range(c["Hkv"]):
            k = s["k_cache"][pages, h].reshape(-1, c["D"])[:length].double()
            v = s["v_cache"][pages, h].reshape(-1, c["D"])[:length].double()
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


def _exact_rope(s):
    c, R = s["case"], s["case"]["rot"]
    pair = torch.arange(R // 2, dtype=torch.float64, device=DEV)
    freq = torch.exp(pair * (-2.0 * math.log(THETA) / R))
    gain = 1.0
    if c["factor"] != 1.0:
        # a pair keeps its frequency above 32 turns in 32768 positions, is slowed by the factor below one turn
        edge = [R / 2 * math.log(32768 / (2 * math.pi * turns)) / math.log(THETA) for turns in (32.0, 1.0)]
        lo, hi = max(math.floor(edge[0]), 0), min(math.ceil(edge[1]), R - 1)
        slow = torch.clamp((pair - lo) / max(hi - lo, 1e-3), 0, 1)
        freq = freq * (1 - slow + slow / c["factor"])
        gain = 1 + 0.1 * math.log(c["factor"])
    turn = torch.polar(torch.full((c["N"], R // 2), gain, dtype=torch.float64, device=DEV),
                       torch.outer(s["positions"].double(), freq))[:, None]

    def rotated(x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["D"] + 1e-6) * w.double()
        if c["interleaved"]:
            z = torch.view_as_complex(x[..., :R].reshape(*x.shape[:-1], R // 2, 2).contiguous()) * turn
            r = torch.view_as_real(z).reshape(*x.shape[:-1], R)
        else:
            z = torch.complex(x[..., :R // 2], x[..., R // 2:R]) * turn
            r = torch.cat([z.real, z.imag], -1)
        return torch.cat([r, x[..., R:]], -1)

    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    flat = lambda cache: cache.transpose(1, 2).reshape(-1, c["Hkv"], c["D"])  # noqa: E731
    k2, v2 = flat(kc).clone(), flat(vc).clone()
    k2[s["slots"]], v2[s["slots"]] = rotated(s["k"], s["k_weight"]), s["v"].double()
    back = lambda x: x.view(-1, c["ps"], c["Hkv"], c["D"]).transpose(1, 2).contiguous()  # noqa: E731
    return {"q": rotated(s["q"], s["q_weight"]), "k_cache": back(k2), "v_cache": back(v2)}


def exact(case, seed):
    if case["op"] == "pages":
        return None     # whole numbers: there is nothing to be computed in 64 bits
    if case["op"] == "attn" and case["B"] * case["Hkv"] * case["n_q"] > 20000:
        return None
    s = prepare(case, seed)
    return _exact_attn(s) if case["op"] == "attn" else _exact_rope(s)
