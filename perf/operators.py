"""Performance cases of the paged-cache operators on one MI355X.

The operators serve requests of different lengths from one pool of cache pages: the plan that
turns request lengths into block tables and slots (``apex_paged_plan``), the store of new keys
and values into their pages (``apex_paged_store``) and the attention of new tokens over the pages
(``apex_attention_paged``).  With ``own`` the calls are the library's; without, the same is
computed from elementary torch operations in 32 bits (the plan in whole numbers), rounded once.

Head shapes are those of the workload table in ``paper_2608_11688_amd.configs`` (Granite-1B 16
query heads and 8 key/value heads of 64, Granite-3B 24 and 8 of 64, OLMoE 16 and 16 of 128, Mixtral
32 and 8 of 128); ``draw`` spreads requests, chunks, contexts, page sizes, groupings, formats,
windows and sinks over the ranges between and around them.  A case's request lengths follow from
the case alone, its values and the order of its pages from the seed.
"""
import math
import random

import torch

own = False   # whether run() makes the library's calls

DEV = "cuda"


# ------------------------------------------------------------------------------ cases
def _plan(name, R, new, ctx, page, ended=0, long=0, pad=0):
    """R requests; `long` of them bring a chunk of up to `new` tokens, the others one; every
    `ended`-th has ended (0: none); `pad` rows of the slot map behind the last token."""
    return dict(name=name, kind="plan", R=R, new=new, ctx=ctx, page=page, ended=ended, long=long, pad=pad)


def _store(name, T, G, hd, page, dtype, fmt, pad=0):
    return dict(name=name, kind="store", T=T, G=G, hd=hd, page=page, dtype=dtype, fmt=fmt, pad=pad)


def _attn(name, R, new, ctx, heads, page, dtype="bf16", fmt="bf16", long=None, window=0, sinks=0, pad=0):
    H, G, hd = heads
    return dict(name=name, kind="attn", R=R, new=new, ctx=ctx, H=H, G=G, hd=hd, page=page, dtype=dtype,
                fmt=fmt, long=R if long is None else long, window=window, sinks=sinks, pad=pad)


GRANITE_1B, GRANITE_3B, OLMOE, MIXTRAL = (16, 8, 64), (24, 8, 64), (16, 16, 128), (32, 8, 128)


def listed():
    return [
        # a decode step of 32 users: every request brings one token, few need a page; latency
        _plan("plan_decode_r32", 32, 1, 2000, 16),
        # a busy server's step: 1024 requests, prompts among them, every 16th ends
        _plan("plan_mixed_r1024", 1024, 512, 8192, 32, ended=16, long=48, pad=100),
        # the new keys and values of one decode step of 32 users
        _store("store_decode_bf16", 32, 8, 128, 16, "bf16", "bf16"),
        # a prompt chunk into an 8-bit cache, activations of 32 bits as the framework's own
        _store("store_chunk_fp8", 8192, 8, 128, 64, "fp32", "fp8", pad=61),
        # a single user's token, a short context: the launches count
        _attn("attn_one_token", 1, 1, 1024, GRANITE_1B, 16),
        # a batch of users at different lengths, 32-bit activations: the stream of keys and values
        _attn("attn_decode_r32_fp32", 32, 1, 4000, MIXTRAL, 16, dtype="fp32"),
        # four very long contexts in an 8-bit cache: few rows, work split along the positions
        _attn("attn_decode_long_fp8", 4, 1, 131072, MIXTRAL, 64, fmt="fp8"),
        # long chats under a sliding window with four sinks: most pages are never read
        _attn("attn_decode_window", 64, 1, 16384, MIXTRAL, 32, window=4096, sinks=4),
        # a chunk of a long prompt, the largest product
        _attn("attn_chunk_mixtral", 1, 4096, 12288, MIXTRAL, 128),
        # ragged chunks of eight prompts over an 8-bit cache, one query head per key/value head
        _attn("attn_chunk_ragged_fp8", 8, 700, 3500, OLMOE, 16, fmt="fp8"),
        # a chunk under a window with sinks, 32-bit activations, heads of 64
        _attn("attn_chunk_window_fp32", 2, 2048, 2100, GRANITE_3B, 32, dtype="fp32", window=1024, sinks=4),
        # what a server runs most: one prompt's chunk among single tokens, a padded batch
        _attn("attn_mixed_batch", 32, 512, 4096, MIXTRAL, 16, long=1, pad=17),
    ]


MOST_FLOPS = 0.9e12     # of a drawn pass
MOST_SCORES = 2.0e9     # requests * query heads * longest chunk * longest context
MOST_POSITIONS = 5e5    # cached positions of all requests


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["plan", "store", "attn", "attn", "attn", "attn"])
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "plan":
        R = _log_int(rng, 1, 1024)
        return dict(kind="plan", R=R, new=_log_int(rng, 1, 512), ctx=_log_int(rng, 1, 8192), page=page,
                    ended=rng.choice([0, 0, 3, 16]), long=rng.randint(0, min(R, 64)), pad=rng.randint(0, 100))
    if kind == "store":
        return dict(kind="store", T=_log_int(rng, 1, 8192), G=rng.choice([1, 2, 3, 8, 16]),
                    hd=rng.choice([64, 128]), page=page, dtype=rng.choice(["fp32", "bf16"]),
                    fmt=rng.choice(["bf16", "fp8"]), pad=rng.randint(0, 64))
    while True:
        R = _log_int(rng, 1, 64)
        chunk = rng.random() < 0.6
        G, per = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 3, 4, 4, 5, 8])
        c = dict(kind="attn", R=R, new=_log_int(rng, 2, 4096) if chunk else 1,
                 ctx=_log_int(rng, 1, 16384 if chunk else 131072), H=G * per, G=G, hd=rng.choice([64, 128]),
                 page=page, dtype=rng.choice(["bf16", "bf16", "fp32"]), fmt=rng.choice(["bf16", "fp8"]),
                 long=rng.choice([1, R]) if chunk else R, window=rng.choice([0, 0, _log_int(rng, 1, 4096)]),
                 sinks=rng.choice([0, 4, 17]), pad=rng.randint(0, 20))
        if c["H"] > 64:
            continue
        cached, new = _lengths(c)
        if (work(c)["flops"] <= MOST_FLOPS and sum(cached) * G <= MOST_POSITIONS * 8
                and R * c["H"] * max(new) * (max(cached) + max(new)) <= MOST_SCORES):
            return c


def _lengths(case):
    """Cached and new positions of every request (-1: the request has ended), from the case alone."""
    rng = random.Random("%d %d %d %d" % (case["R"], case["new"], case["ctx"], case["page"]))
    R = case["R"]
    cached = [rng.randint(case["ctx"] // 4, case["ctx"]) for _ in range(R)]
    cached[rng.randrange(R)] = case["ctx"]
    chunks = set(rng.sample(range(R), case["long"]))
    new = [rng.randint(max(1, case["new"] // 4), case["new"]) if r in chunks else 1 for r in range(R)]
    if case["long"]:
        new[min(chunks)] = case["new"]
    if case.get("ended"):
        new = [-1 if r % case["ended"] == case["ended"] - 1 else n for r, n in enumerate(new)]
    return cached, new


def _blocks(n, page):
    return (n + page - 1) // page


# ------------------------------------------------------------------------------ states
def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _pool(case, n_pages, gen):
    """Pages of keys or values and the scales of their rows (E4M3 only)."""
    shape = (n_pages, case["G"], case["page"], case["hd"])
    x = torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)
    if case["fmt"] == "bf16":
        return x, None
    s = torch.rand(shape[:3], generator=gen, device=DEV) * 0.004 + 0.004     # of rows of size one
    return (x * 100).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), s


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case)
    page = case["page"]
    if case["kind"] == "store":
        T, G, hd, pad = case["T"], case["G"], case["hd"], case["pad"]
        n_pages = _blocks(T, page) + 3
        s["k_pages"], s["k_scales"] = _pool(case, n_pages, gen)
        s["v_pages"], s["v_scales"] = _pool(case, n_pages, gen)
        # keys and values as a fused projection leaves them: side by side in a row
        kv = torch.randn(T + pad, 2 * G * hd, generator=gen, device=DEV).to(TYPES[case["dtype"]])
        s["k"], s["v"] = kv[:, :G * hd], kv[:, G * hd:]
        order = torch.randperm(n_pages, generator=gen, device=DEV)
        at = torch.arange(T, device=DEV) + 1     # the first position of its page is taken
        slots = torch.full((T + pad,), -1, dtype=torch.int32, device=DEV)
        slots[:T] = (order[at // page] * page + at % page).int()
        s["slots"], s["n_pages"] = slots, n_pages
        return s
    cached, new = _lengths(case)
    R = case["R"]
    total = sum(n for n in new if n > 0)
    s["T"] = total + case["pad"]
    s["nb"] = max(_blocks(c + max(n, 0), page) for c, n in zip(cached, new)) + 1
    if case["kind"] == "plan":
        held = [_blocks(c, page) for c in cached]
        need = sum(_blocks(c + n, page) - h for c, n, h in zip(cached, new, held) if n > 0)
        s["n_pages"] = n_pages = sum(held) + need + 5
        order = torch.randperm(n_pages, generator=gen, device=DEV).int()
        cols = torch.arange(s["nb"], device=DEV)
        h = torch.tensor(held, device=DEV)
        at = (h.cumsum(0) - h)[:, None] + cols
        s["table"] = torch.where(cols < h[:, None], order[at.clamp(max=n_pages - 1)], -1).int().contiguous()
        s["free"] = torch.cat([order[sum(held):], torch.full((sum(held),), -1, device=DEV).int()])
        s["free_count"] = _int32([n_pages - sum(held)])
        s["cached"], s["new_tokens"] = _int32(cached), _int32(new)
        for name, n in (("seq_len", R), ("cu_new", R + 1), ("slots", s["T"]), ("positions", s["T"]),
                        ("free_out", 1), ("status", R)):
            s[name] = torch.zeros(n, dtype=torch.int32, device=DEV)
        return s
    blocks = [_blocks(c + n, page) for c, n in zip(cached, new)]
    s["n_pages"] = n_pages = sum(blocks) + 2
    s["k_pages"], s["k_scales"] = _pool(case, n_pages, gen)
    s["v_pages"], s["v_scales"] = _pool(case, n_pages, gen)
    order = torch.randperm(n_pages, generator=gen, device=DEV).int()
    cols, b = torch.arange(s["nb"], device=DEV), torch.tensor(blocks, device=DEV)
    at = (b.cumsum(0) - b)[:, None] + cols
    s["table"] = torch.where(cols < b[:, None], order[at.clamp(max=n_pages - 1)], -1).int().contiguous()
    s["seq_len"] = _int32([c + n for c, n in zip(cached, new)])
    cu = [0]
    cu.extend(sum(new[:r + 1]) for r in range(R))
    s["cu_new"], s["max_new"] = _int32(cu), max(new)
    H, hd = case["H"], case["hd"]
    # queries as a fused projection leaves them: in front of the row's keys and values
    wide = torch.randn(s["T"], (H + 2 * case["G"]) * hd, generator=gen, device=DEV)
    wide = (2 * wide).to(TYPES[case["dtype"]])     # scores of size two: some positions stand out
    s["q"] = wide[:, :H * hd]
    s["out"] = torch.zeros(s["T"], H * hd, dtype=TYPES[case["dtype"]], device=DEV)
    return s


# ------------------------------------------------------------------------------ one pass
def run(s):
    if own:
        return _run_own(s)
    return {"plan": _plain_plan, "store": _plain_store, "attn": _plain_attention}[s["kind"]](s)


def _plan_outputs(s, **new):
    names = ("table", "free", "free_out", "seq_len", "cu_new", "slots", "positions", "status")
    return {n: new.get(n, s[n]) for n in names}


def _store_outputs(s):
    if s["fmt"] == "bf16":
        return {"k": s["k_pages"], "v": s["v_pages"]}
    f8 = torch.float8_e4m3fn
    return {"k": s["k_pages"].view(f8), "v": s["v_pages"].view(f8), "k_scales": s["k_scales"],
            "v_scales": s["v_scales"]}


def _run_own(s):
    from paper_2608_11688_amd import native
    if s["kind"] == "plan":
        native.apex_paged_plan(s["cached"], s["new_tokens"], s["R"], s["page"], s["n_pages"], s["nb"], s["T"],
                               s["free"], s["free_count"], s["table"], s["seq_len"], s["cu_new"], s["slots"],
                               s["positions"], s["free_out"], s["status"])
        return _plan_outputs(s)
    if "cache" not in s:   # a program's handle on its pool, made once
        s["cache"] = native.paged_cache(s["fmt"], s["G"], s["hd"], s["page"], s["n_pages"], s["k_pages"],
                                        s["v_pages"], s["k_scales"], s["v_scales"])
    if s["kind"] == "store":
        native.apex_paged_store(s["cache"], s["k"], s["v"], s["dtype"], s["k"].shape[0], s["k"].stride(0),
                                s["v"].stride(0), s["slots"])
        return _store_outputs(s)
    if "workspace" not in s:   # kept by the program for all its calls
        n = native.apex_attention_paged_workspace_bytes(s["T"], s["R"], s["H"], s["G"], s["hd"])
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    native.apex_attention_paged(s["cache"], s["q"], s["dtype"], s["T"], s["R"], s["H"], s["q"].stride(0),
                                s["cu_new"], s["seq_len"], s["table"], s["nb"], s["window"], s["sinks"],
                                s["hd"] ** -0.5, s["out"], s["out"].stride(0), s["workspace"],
                                s["workspace"].numel())
    return s["out"]


def _plain_plan(s):
    page, nb, T, R, n_pages = s["page"], s["nb"], s["T"], s["R"], s["n_pages"]
    cached, new, table = s["cached"].long(), s["new_tokens"].long(), s["table"].long()
    free_count = s["free_count"].long().clamp(0, n_pages)
    valid = (cached >= 0) & (new >= -1) & (cached + new.clamp(min=0) <= nb * page)
    held = (cached.clamp(min=0) + page - 1) // page
    ended = valid & (new == -1)
    given = torch.where(ended, held, 0)
    want = torch.where(valid & (new > 0), new, 0)
    need = torch.where(want > 0, (cached + want + page - 1) // page - held, 0)
    top = torch.minimum(free_count + given.sum(), torch.full_like(free_count, n_pages))
    need_sum = need.cumsum(0)
    fits = (need_sum <= top) & (want.cumsum(0) <= T)
    got = torch.where(fits, want, 0)
    cu = torch.cat([torch.zeros_like(top), got.cumsum(0)])
    # the stack of free pages with those of the ended requests on it
    given_sum = given.cumsum(0)
    at = torch.arange(n_pages, device=DEV)
    k = (at - free_count).clamp(min=0)
    r = torch.searchsorted(given_sum, k, right=True).clamp(max=R - 1)
    back = table[r, (k - (given_sum - given)[r]).clamp(0, nb - 1)]
    stack = torch.where((at >= free_count) & (at < top), back, s["free"].long())
    cols = torch.arange(nb, device=DEV)
    j = (need_sum - need)[:, None] + cols - held[:, None]      # number of a page among those taken
    fresh = (cols >= held[:, None]) & (cols < (cached + got + page - 1)[:, None] // page) & (got > 0)[:, None]
    table = torch.where(fresh, stack[(top - 1 - j).clamp(0, n_pages - 1)], table)
    t = torch.arange(T, device=DEV)
    r = torch.searchsorted(cu[1:], t, right=True).clamp(max=R - 1)
    p = cached[r] + t - cu[r]
    live = t < cu[-1]
    pid = table[r, (p // page).clamp(0, nb - 1)]
    slots = torch.where(live & (pid >= 0) & (pid < n_pages), pid * page + p % page, -1)
    status = torch.where(~valid, 3, torch.where(ended, 1, torch.where(fits | (want == 0), 0, 2)))
    seq_len = torch.where(ended, 0, cached.clamp(0, nb * page) + got)
    taken = torch.where(got > 0, need, 0).sum()
    return _plan_outputs(s, table=table.int(), free=stack.int(), free_out=(top - taken).int(),
                         seq_len=seq_len.int(), cu_new=cu.int(), slots=slots.int(),
                         positions=torch.where(live, p, -1).int(), status=status.int())


def _plain_store(s):
    G, hd, page = s["G"], s["hd"], s["page"]
    slot = s["slots"].long()
    live = (slot >= 0) & (slot < s["n_pages"] * page)
    row = torch.where(live, torch.arange(slot.numel(), device=DEV), 0)   # rows without a slot repeat row 0
    slot = slot[row]
    at = (slot // page, slice(None), slot % page)

    def put(x, pages, scales):
        x = x.reshape(-1, G, hd)[row].float()
        if scales is None:
            pages[at] = x.to(torch.bfloat16)
            return
        peak = x.abs().amax(-1)
        scale = peak / torch.full_like(peak, 448.0)
        q = torch.where(scale[..., None] > 0, x / scale[..., None], 0.0).clamp(-448.0, 448.0)
        pages[at] = q.to(torch.float8_e4m3fn).view(torch.uint8)
        scales[at] = scale

    put(s["k"], s["k_pages"], s["k_scales"])
    put(s["v"], s["v_pages"], s["v_scales"])
    return _store_outputs(s)


def _plain_attention(s):
    R, T, H, G, hd, n, page = s["R"], s["T"], s["H"], s["G"], s["hd"], s["max_new"], s["page"]
    per, L = H // G, s["nb"] * page
    cu, seq = s["cu_new"].long(), s["seq_len"].long()
    new = cu[1:] - cu[:-1]
    i = torch.arange(n, device=DEV)
    q = s["q"][(cu[:-1, None] + i).clamp(max=T - 1)].float()               # [R, n, H hd]
    q = q.view(R, n, G, per, hd).permute(0, 2, 1, 3, 4).reshape(R, G, n * per, hd)
    ids = s["table"].long()
    good = (ids >= 0) & (ids < s["n_pages"])
    ids = torch.where(good, ids, 0)

    def gathered(pages, scales):                                           # [R, G, L, hd]
        if scales is None:
            x = pages[ids].float()
        else:
            x = pages.view(torch.float8_e4m3fn).float()[ids] * scales[ids][..., None]
        return x.permute(0, 2, 1, 3, 4).reshape(R, G, L, hd)

    score = torch.matmul(q, gathered(s["k_pages"], s["k_scales"]).transpose(2, 3).contiguous())
    score = score.mul_(hd ** -0.5).view(R, G, n, per, L)
    p = (seq - new)[:, None, None] + i[:, None]                            # [R, n, 1]
    j = torch.arange(L, device=DEV)
    seen = (j <= p) & good.repeat_interleave(page, 1)[:, None]
    if s["window"]:
        seen &= (j > p - s["window"]) | (j < s["sinks"])
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = score.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = weight.sum(-1)
    out = torch.matmul(weight.view(R, G, n * per, L), gathered(s["v_pages"], s["v_scales"]))
    out = out / torch.where(total > 0, total, 1.0).view(R, G, n * per, 1)
    out = out.view(R, G, n, per, hd).permute(0, 2, 1, 3, 4).reshape(R, n, H * hd)
    t = torch.arange(T, device=DEV)
    r = torch.searchsorted(cu[1:], t, right=True).clamp(max=R - 1)
    rows = out[r, (t - cu[r]).clamp(0, n - 1)].to(s["out"].dtype)
    return torch.where((t < cu[-1])[:, None], rows, s["out"])


# ------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    if case["kind"] == "plan":
        return None
    s = prepare(case, seed)
    if case["kind"] == "store":
        return _exact_store(s)
    T, H, G, hd, page, window, sinks = (s[k] for k in ("T", "H", "G", "hd", "page", "window", "sinks"))
    out = s["out"].double()
    cu, seq, table = s["cu_new"].tolist(), s["seq_len"].tolist(), s["table"].tolist()
    q = s["q"].double().reshape(T, G, H // G, hd)
    for r in range(case["R"]):
        rows, end = cu[r + 1] - cu[r], seq[r]
        ids = torch.tensor(table[r][:_blocks(end, page)], device=DEV)

        def values(pages, scales, g):
            x = pages[ids, g]
            if scales is None:
                return x.double().reshape(-1, hd)[:end]
            return (x.view(torch.float8_e4m3fn).float().double() * scales[ids, g].double()[..., None]).reshape(-1, hd)[:end]

        for g in range(G):
            K, V = values(s["k_pages"], s["k_scales"], g), values(s["v_pages"], s["v_scales"], g)
            for lo in range(0, rows, 1024):
                hi = min(rows, lo + 1024)
                at = torch.arange(end - rows + lo, end - rows + hi, device=DEV)
                first = torch.zeros_like(at) if not window else (at - window + 1).clamp(min=0)
                pos = torch.arange(end, device=DEV)
                hidden = (pos > at[:, None]) | ((pos < first[:, None]) & (pos >= sinks))
                for h in range(H // G):
                    logit = (q[cu[r] + lo:cu[r] + hi, g, h] @ K.T) / math.sqrt(hd)
                    logit[hidden] = -math.inf
                    col = (g * (H // G) + h) * hd
                    out[cu[r] + lo:cu[r] + hi, col:col + hd] = torch.softmax(logit, -1) @ V
    return out


def _exact_store(s):
    G, hd, page = s["G"], s["hd"], s["page"]
    T = s["T"]
    slots = s["slots"][:T].long()
    found = {}
    for name in ("k", "v"):
        x = s[name][:T].double().reshape(T, G, hd)
        pages, scales = s[name + "_pages"], s[name + "_scales"]
        if scales is None:
            y = pages.double()
            # bf16 keeps 8 significant bits; ties go to the even one
            m, e = torch.frexp(x)
            y[slots // page, :, slots % page] = torch.ldexp((m * 256).round(), e - 8)
            found[name] = y
            continue
        scale = (x.abs().amax(-1) / 448.0).float().double()
        ratio = x / torch.where(scale > 0, scale, 1.0)[..., None]
        # E4M3 keeps 4 significant bits, steps of 2^-9 at least
        step = torch.exp2(torch.frexp(ratio)[1].double() - 4).clamp(min=2.0 ** -9)
        y, z = pages.view(torch.float8_e4m3fn).float().double(), scales.double()
        y[slots // page, :, slots % page] = ((ratio / step).round() * step).clamp(-448.0, 448.0)
        z[slots // page, :, slots % page] = scale
        found[name], found[name + "_scales"] = y, z
    return found


# ------------------------------------------------------------------------------ what a pass cannot do without
def _visible(cached, new, window, sinks):
    """Pairs of a new token and a position it sees, and the positions that any of them sees."""
    if not window:
        return new * cached + new * (new + 1) // 2, cached + new
    pairs = 0
    for p in range(cached, cached + new):
        low = max(0, p - window + 1)
        pairs += p - low + 1 + min(sinks, low)
    low = max(0, cached - window + 1)
    return pairs, cached + new - low + min(sinks, low)


def work(case):
    if case["kind"] == "store":
        n = 2 * case["T"] * case["G"]
        size_in, size_out = (4 if case["dtype"] == "fp32" else 2), (2 if case["fmt"] == "bf16" else 1)
        scales = 4 if case["fmt"] == "fp8" else 0
        return {"bytes": n * (case["hd"] * (size_in + size_out) + scales) + 4 * (case["T"] + case["pad"]), "flops": 0}
    cached, new = _lengths(case)
    page = case["page"]
    if case["kind"] == "plan":
        T = sum(n for n in new if n > 0) + case["pad"]
        pages = sum(_blocks(c + n, page) - _blocks(c, page) if n > 0 else _blocks(c, page) if n < 0 else 0
                    for c, n in zip(cached, new))
        return {"bytes": 8 * T + 8 * pages + 20 * case["R"], "flops": 0}
    seen = [_visible(c, n, case["window"], case["sinks"]) for c, n in zip(cached, new)]
    row = case["hd"] * (2 if case["fmt"] == "bf16" else 1) + (4 if case["fmt"] == "fp8" else 0)
    size = 4 if case["dtype"] == "fp32" else 2
    positions = sum(x[1] for x in seen)
    return {"bytes": 2 * positions * case["G"] * row + 2 * sum(new) * case["H"] * case["hd"] * size
            + 4 * sum(_blocks(x[1], page) for x in seen),
            "flops": 4 * case["hd"] * case["H"] * sum(x[0] for x in seen)}
