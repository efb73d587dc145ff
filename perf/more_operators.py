"""Performance cases of the operators between the residual stream and the paged cache, on one MI355X.

A step's attention block is: projection of the activations to queries, keys and values by weights of
4 bits with a scale and a zero point per group (``apex_linear_w4``), rotary positions of queries and
keys with the keys and values stored into their pages on the way (``apex_paged_store_rotary``; alone:
``apex_rotary``), attention, projection back with the residual added (``apex_linear_w4`` again).
With ``own`` the calls are the library's; without, the same is computed from elementary torch
operations in 32 bits (angles in 64), rounded once.

Sizes are those of the workload table in ``paper_2608_11688_amd.configs`` (Granite-1B hidden size 1024,
16 query heads and 8 key/value heads of 64; Mixtral 4096, 32 and 8 of 128) or generic; ``draw`` spreads
rows, sizes, groups, types, head shapes and layouts over the ranges between and around them.

Packed weights [N, K] of 4 bits: rows of K rounded up to 128 codes (0 behind K), 64 bytes for every 128,
in which the 32-bit word 4 a + j holds the codes of k = 32 j + 8 a + e, e = 0..7, at the bits
4 (e / 2) + 16 (e mod 2); then for every group of `group` codes along k a 32-bit word per row, the
scale as bf16 in the upper half and the zero point as bf16 in the lower: weight = s * (q - z).
"""
import math

import torch

own = False   # whether run() makes the library's calls

DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------ cases
def _linear(name, T, N, K, group, x="bf16", y="bf16", bias=False, residual=False):
    return dict(name=name, kind="linear", T=T, N=N, K=K, group=group, x=x, y=y, bias=bias, residual=residual)


def _rotary(name, T, heads, hd, dim, layout, dtype, pos, factor=1.0, pad=0):
    """`heads` heads of `hd` of which the first `dim` turn; positions up to `pos`; frequencies
    divided by `factor`."""
    return dict(name=name, kind="rotary", T=T, heads=heads, hd=hd, dim=dim, layout=layout, dtype=dtype, pos=pos,
                factor=factor, pad=pad)


def _store(name, T, H, G, hd, dim, layout, dtype, fmt, page, pos, factor=1.0, pad=0):
    return dict(name=name, kind="store", T=T, H=H, G=G, hd=hd, dim=dim, layout=layout, dtype=dtype, fmt=fmt, page=page,
                pos=pos, factor=factor, pad=pad)


def listed():
    return [
        # one user's token, the smallest fused projection (32 heads of 64): latency
        _linear("linear_token_small", 1, 2048, 1024, 64, x="fp32", y="fp32"),
        # one user's token, 48 heads of 128: the stream of the weights
        _linear("linear_token_qkv", 1, 6144, 4096, 128, x="fp32"),
        # four users' tokens through a wide projection, small groups: the longest stream of weights
        _linear("linear_wide_t4", 4, 32768, 4096, 32),
        # odd sizes: seven tokens, a row that ends inside a block of codes, a bias
        _linear("linear_ragged_t7", 7, 1031, 1416, 32, bias=True),
        # 32 users' tokens back into the residual stream
        _linear("linear_out_r32", 32, 4096, 4096, 64, y="fp32", residual=True),
        # a hundred rows of 32 bits: between the stream of weights and the matrix product
        _linear("linear_t100_fp32", 100, 6144, 4096, 128, x="fp32", y="fp32"),
        # a prompt's chunk: the matrix product
        _linear("linear_chunk", 2048, 6144, 4096, 128),
        # queries and keys of 32 users' tokens: a launch
        _rotary("rotary_decode_r32", 32, 40, 128, 128, "half", "bf16", 100000),
        # a long chunk far behind, half of each head turned in neighbouring pairs, 32 bits, positions interpolated
        _rotary("rotary_chunk_part_fp32", 8192, 32, 64, 32, "interleaved", "fp32", 131072, factor=8.0, pad=5),
        # the new tokens of 32 users into a bf16 cache
        _store("store_rotary_decode", 32, 32, 8, 128, 128, "half", "bf16", "bf16", 16, 100000),
        # a long chunk into an 8-bit cache, activations of 32 bits, a padded batch
        _store("store_rotary_chunk_fp8", 8192, 32, 8, 128, 128, "half", "fp32", "fp8", 64, 131072, pad=61),
    ]


MOST_FLOPS = 1.04e11    # of a drawn product
MOST_WEIGHTS = 1.4e8    # codes of a drawn product
MOST_VALUES = 4.0e7     # of drawn rows of queries, keys and values


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "rotary", "store"])
    while True:
        if kind == "linear":
            K = rng.choice([8 * _log_int(rng, 8, 1024), 128 * _log_int(rng, 1, 64)])
            c = dict(kind="linear", T=rng.choice([_log_int(rng, 1, 64), _log_int(rng, 1, 2048)]),
                     N=_log_int(rng, 16, 32768), K=K, group=rng.choice([32, 64, 128]),
                     x=rng.choice(["fp32", "bf16", "bf16"]), y=rng.choice(["fp32", "bf16"]),
                     bias=rng.random() < 0.3, residual=rng.random() < 0.4)
            if 2.0 * c["T"] * c["N"] * K <= MOST_FLOPS and c["N"] * K <= MOST_WEIGHTS:
                return c
            continue
        hd = rng.choice([64, 128])
        c = dict(kind=kind, T=_log_int(rng, 1, 8192), hd=hd, dim=rng.choice([hd, hd, hd // 2, 48]),
                 layout=rng.choice(["half", "interleaved"]), dtype=rng.choice(["fp32", "bf16"]),
                 pos=_log_int(rng, 16, 1000000), factor=rng.choice([1.0, 4.0, 32.0]), pad=rng.randint(0, 64))
        G, per = rng.choice([1, 2, 3, 8, 16]), rng.choice([1, 2, 4, 5, 8])
        if kind == "rotary":
            c.update(heads=G * (per + 1))
            heads = c["heads"]
        else:
            c.update(H=G * per, G=G, fmt=rng.choice(["bf16", "fp8"]), page=rng.choice([16, 32, 64, 128, 256]))
            heads = G * (per + 2)
        if c["T"] * heads * hd <= MOST_VALUES:
            return c


# ------------------------------------------------------------------------------ states
LOW, HIGH = (0, 4, 1, 5), (2, 6, 3, 7)   # elements of a word's 8 codes in the nibbles of its bytes


def _blocks(n, size):
    return (n + size - 1) // size


def _pack(codes, scales, zeros):
    """codes uint8 [N, K128]; scales, zeros bf16 [N, K128 / group]: the packed weights, uint8."""
    N = codes.shape[0]
    c = codes.view(N, -1, 4, 4, 8).transpose(2, 3)
    c = (c[..., LOW] | c[..., HIGH] << 4).contiguous().view(-1)
    words = torch.stack([zeros.t(), scales.t()], -1).contiguous()    # [groups, N, 2]
    return torch.cat([c, words.view(torch.uint8).view(-1)])


def _unpack(s):
    """(q [N, K] uint8, scales, zeros [N, groups] bf16) of a state's packed weights."""
    N, K, group = s["N"], s["K"], s["group"]
    nb = _blocks(K, 128)
    n = N * nb * 64
    c = s["w"][:n].view(N, nb, 4, 4, 4)
    q = torch.empty(N, nb, 4, 4, 8, dtype=torch.uint8, device=DEV)
    q[..., LOW], q[..., HIGH] = c & 15, c >> 4
    q = q.transpose(2, 3).reshape(N, nb * 128)[:, :K]
    words = s["w"][n:].view(torch.bfloat16).view(nb * 128 // group, N, 2)
    return q, words[..., 1].t(), words[..., 0].t()


def _prepare_linear(case, gen):
    s = dict(case)
    T, N, K, group = (case[k] for k in ("T", "N", "K", "group"))
    K128 = _blocks(K, 128) * 128
    groups = K128 // group
    # weights of size 1 / sqrt(K) as a quantiser leaves them: zero points near the middle
    zeros = torch.randint(5, 11, (N, groups), generator=gen, device=DEV).to(torch.bfloat16)
    scales = ((torch.rand(N, groups, generator=gen, device=DEV) + 0.5) * 0.36 * K ** -0.5).to(torch.bfloat16)
    q = torch.empty(N, groups, group, dtype=torch.bfloat16, device=DEV).normal_(generator=gen).mul_(2.7)
    q = (q + zeros[..., None]).round_().clamp_(0, 15).to(torch.uint8).view(N, K128)
    q[:, K:] = 0
    s["w"] = _pack(q, scales, zeros)
    s["xs"] = torch.randn(T, K, generator=gen, device=DEV).to(TYPES[case["x"]])
    s["b"] = torch.randn(N, generator=gen, device=DEV) if case["bias"] else None
    s["r"] = torch.randn(T, N, generator=gen, device=DEV).to(TYPES[case["y"]]) if case["residual"] else None
    s["out"] = torch.zeros(T, N, dtype=TYPES[case["y"]], device=DEV)
    return s


def _positions(case, gen):
    """Positions of T tokens, -1 behind the last."""
    p = torch.randint(0, case["pos"] + 1, (case["T"],), generator=gen, device=DEV, dtype=torch.int32)
    p[0] = case["pos"]
    return torch.cat([p, torch.full((case["pad"],), -1, dtype=torch.int32, device=DEV)])


def _frequencies(case):
    i = torch.arange(case["dim"] // 2, dtype=torch.float64, device=DEV)
    return 10000.0 ** (-2.0 * i / case["dim"]) / case["factor"]


def _amplitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0


def _pool(case, n_pages, gen):
    """Pages of keys or values and the scales of their rows (E4M3 only)."""
    shape = (n_pages, case["G"], case["page"], case["hd"])
    x = torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)
    if case["fmt"] == "bf16":
        return x, None
    scales = torch.rand(shape[:3], generator=gen, device=DEV) * 0.004 + 0.004
    return (x * 100).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), scales


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    if case["kind"] == "linear":
        return _prepare_linear(case, gen)
    s = dict(case)
    s["positions"], s["freq"], s["amplitude"] = _positions(case, gen), _frequencies(case), _amplitude(case)
    rows, dtype, hd = case["T"] + case["pad"], TYPES[case["dtype"]], case["hd"]
    if case["kind"] == "rotary":
        # queries and keys in front of the values of a fused projection's row
        wide = torch.randn(rows, (case["heads"] + 2) * hd, generator=gen, device=DEV).to(dtype)
        s["xs"] = wide[:, :case["heads"] * hd]
        s["out"] = torch.zeros(rows, case["heads"] * hd, dtype=dtype, device=DEV)
        return s
    T, H, G, page = (case[k] for k in ("T", "H", "G", "page"))
    n_pages = _blocks(T + 1, page) + 3
    s["k_pages"], s["k_scales"] = _pool(case, n_pages, gen)
    s["v_pages"], s["v_scales"] = _pool(case, n_pages, gen)
    wide = torch.randn(rows, (H + 2 * G) * hd, generator=gen, device=DEV).to(dtype)
    s["q"], s["k"], s["v"] = wide[:, :H * hd], wide[:, H * hd:(H + G) * hd], wide[:, (H + G) * hd:]
    s["q_out"] = torch.zeros(rows, H * hd, dtype=dtype, device=DEV)
    order = torch.randperm(n_pages, generator=gen, device=DEV)
    at = torch.arange(T, device=DEV) + 1     # the first position of its page is taken
    slots = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    slots[:T] = (order[at // page] * page + at % page).int()
    s["slots"], s["n_pages"] = slots, n_pages
    return s


# ------------------------------------------------------------------------------ one pass
def run(s):
    if own:
        return _run_own(s)
    return {"linear": _plain_linear, "rotary": _plain_rotary, "store": _plain_store}[s["kind"]](s)


def _store_outputs(s, q):
    out = {"q": q, "k": s["k_pages"], "v": s["v_pages"]}
    if s["fmt"] == "fp8":
        f8 = torch.float8_e4m3fn
        out.update(k=s["k_pages"].view(f8), v=s["v_pages"].view(f8), k_scales=s["k_scales"], v_scales=s["v_scales"])
    return out


def _run_own(s):
    from paper_2608_11688_amd import native
    if s["kind"] == "linear":
        T, N, K, group = s["T"], s["N"], s["K"], s["group"]
        if "workspace" not in s:   # kept by the program for all its calls
            n = native.apex_linear_w4_workspace_bytes(T, N, K, group, s["x"])
            s["workspace"] = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)
        x, y, r = s["xs"], s["out"], s["r"]
        native.apex_linear_w4(s["w"], N, K, group, x, s["x"], T, x.stride(0), s["b"], r, r.stride(0) if r is not None else 0,
                              y, s["y"], y.stride(0), s["workspace"], s["workspace"].numel())
        return y
    if "rotation" not in s:   # a program's descriptor of its positions, made once
        s["rotation"] = native.rotary(s["layout"], s["dim"], s["freq"], s["amplitude"])
    if s["kind"] == "rotary":
        x, y = s["xs"], s["out"]
        native.apex_rotary(s["rotation"], x, s["dtype"], x.shape[0], s["heads"], s["hd"], x.stride(0), s["positions"],
                           y, y.stride(0))
        return y
    if "cache" not in s:   # and its handle on its pool
        s["cache"] = native.paged_cache(s["fmt"], s["G"], s["hd"], s["page"], s["n_pages"], s["k_pages"],
                                        s["v_pages"], s["k_scales"], s["v_scales"])
    q, k, v, y = s["q"], s["k"], s["v"], s["q_out"]
    native.apex_paged_store_rotary(s["cache"], s["rotation"], q, k, v, s["dtype"], q.shape[0], s["H"], q.stride(0),
                                   k.stride(0), v.stride(0), s["slots"], s["positions"], y, y.stride(0))
    return _store_outputs(s, y)


def _plain_linear(s):
    q, scales, zeros = _unpack(s)
    w = scales.float().repeat_interleave(s["group"], 1)[:, :s["K"]]
    w = w * (q.float() - zeros.float().repeat_interleave(s["group"], 1)[:, :s["K"]])
    y = s["xs"].float() @ w.t()
    if s["b"] is not None:
        y = y + s["b"]
    if s["r"] is not None:
        y = y + s["r"].float()
    return y.to(s["out"].dtype)


def _turned(s, x, heads):
    """Rows [T, heads * hd] at their positions, in 32 bits."""
    hd, dim = s["hd"], s["dim"]
    angle = s["positions"].double()[:, None] * s["freq"]
    cos, sin = ((f(angle) * s["amplitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    x = x.reshape(-1, heads, hd).float()
    y = x.clone()
    a, b = (slice(0, dim // 2), slice(dim // 2, dim)) if s["layout"] == "half" else (slice(0, dim, 2), slice(1, dim, 2))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    return y


def _live(s, new, old):
    """Rows of tokens that have a position; the others as they were."""
    return torch.where((s["positions"] >= 0)[:, None], new.reshape(old.shape).to(old.dtype), old)


def _plain_rotary(s):
    return _live(s, _turned(s, s["xs"], s["heads"]), s["out"])


def _plain_store(s):
    G, hd, page = s["G"], s["hd"], s["page"]
    slot = s["slots"].long()
    live = (slot >= 0) & (slot < s["n_pages"] * page) & (s["positions"] >= 0)
    row = torch.where(live, torch.arange(slot.numel(), device=DEV), 0)   # rows without a slot repeat row 0
    slot = slot[row]
    at = (slot // page, slice(None), slot % page)

    def put(x, pages, scales):
        x = x[row]
        if scales is None:
            pages[at] = x.to(torch.bfloat16)
            return
        peak = x.abs().amax(-1)
        scale = peak / torch.full_like(peak, 448.0)
        q = torch.where(scale[..., None] > 0, x / scale[..., None], 0.0).clamp(-448.0, 448.0)
        pages[at] = q.to(torch.float8_e4m3fn).view(torch.uint8)
        scales[at] = scale

    put(_turned(s, s["k"], G), s["k_pages"], s["k_scales"])
    put(s["v"].reshape(-1, G, hd).float(), s["v_pages"], s["v_scales"])
    return _store_outputs(s, _live(s, _turned(s, s["q"], s["H"]), s["q_out"]))


# ------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "linear":
        return _exact_linear(s)
    if case["kind"] == "rotary":
        T = case["T"]
        y = s["out"].double()
        y[:T] = _exact_turned(s, s["xs"][:T], case["heads"]).reshape(T, -1)
        return y
    return _exact_store(s)


def _exact_linear(s):
    T, N, K, group = s["T"], s["N"], s["K"], s["group"]
    nb = _blocks(K, 128)
    words = s["w"][:N * nb * 64].view(torch.int32).long().view(N, nb, 4, 4)      # [row, block, a, j]
    scale_words = s["w"][N * nb * 64:].view(torch.int32).view(-1, N)             # [group, row]
    y = torch.zeros(T, N, dtype=torch.float64, device=DEV)
    x = s["xs"].double()
    for lo in range(0, K, 32):
        hi, g = min(lo + 32, K), lo // group
        word = words[:, lo // 128, :, lo // 32 % 4]                              # the codes of k = lo + 8 a + e
        w = torch.stack([(word >> (4 * (e // 2) + 16 * (e % 2))) & 15 for e in range(8)], -1).double()
        z = (scale_words[g] << 16).view(torch.float32).double()
        t = (scale_words[g] & -65536).view(torch.float32).double()
        w = (w.reshape(N, 32) - z[:, None]) * t[:, None]
        y += x[:, lo:hi] @ w[:, :hi - lo].t().contiguous()
    if s["b"] is not None:
        y += s["b"].double()
    if s["r"] is not None:
        y += s["r"].double()
    return y


def _exact_turned(s, x, heads):
    """A pair as a complex number times e^(i angle)."""
    T, hd, dim = x.shape[0], s["hd"], s["dim"]
    x = x.double().reshape(T, heads, hd)
    angle = s["positions"][:T].double()[:, None, None] * s["freq"]
    turn = torch.polar(torch.full_like(angle, s["amplitude"]), angle)
    if s["layout"] == "half":
        z = torch.complex(x[..., :dim // 2].contiguous(), x[..., dim // 2:dim].contiguous()) * turn
        front = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.view_as_complex(x[..., :dim].reshape(T, heads, dim // 2, 2).contiguous()) * turn
        front = torch.view_as_real(z).reshape(T, heads, dim)
    return torch.cat([front, x[..., dim:]], -1)


def _exact_store(s):
    T, H, G, hd, page = (s[k] for k in ("T", "H", "G", "hd", "page"))
    slots = s["slots"][:T].long()
    q = s["q_out"].double()
    q[:T] = _exact_turned(s, s["q"][:T], H).reshape(T, -1)
    found = {"q": q}
    for name, x in (("k", _exact_turned(s, s["k"][:T], G)), ("v", s["v"][:T].double().reshape(T, G, hd))):
        pages, scales = s[name + "_pages"], s[name + "_scales"]
        if scales is None:
            y = pages.double()
            y[slots // page, :, slots % page] = x
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
SIZES = {"fp32": 4, "bf16": 2, "fp8": 1}


def work(case):
    T = case["T"]
    if case["kind"] == "linear":
        N, K = case["N"], case["K"]
        y = T * N * SIZES[case["y"]]
        return {"bytes": N * _blocks(K, 2) + 4 * N * _blocks(K, case["group"]) + T * K * SIZES[case["x"]]
                + y * (2 if case["residual"] else 1) + (4 * N if case["bias"] else 0), "flops": 2 * T * N * K}
    size, hd, rows = SIZES[case["dtype"]], case["hd"], T + case["pad"]
    if case["kind"] == "rotary":
        return {"bytes": 2 * T * case["heads"] * hd * size + 4 * rows + 4 * case["dim"],
                "flops": 3 * T * case["heads"] * case["dim"]}
    G, H = case["G"], case["H"]
    scales = 8 * T * G if case["fmt"] == "fp8" else 0
    return {"bytes": T * hd * ((2 * H + 2 * G) * size + 2 * G * SIZES[case["fmt"]]) + scales + 8 * rows
            + 4 * case["dim"], "flops": 3 * T * (H + G) * case["dim"]}
