"""Rotary positions and the store with rotation against the float64 oracle.

Tolerances.  A sine or cosine times the amplitude is rounded once to 32 bits from an angle in 64 (2^-25 of the amplitude,
for any position), the smaller of the two products of a turned value and its sum once more, 2^-24 of their size each: a
turned value is off by less than 2^-22 of |amplitude| (|a| + |b|).  Rounding to bf16 adds half a step, 2^-8 of the value.
An E4M3 code is within half a step of the value: 2^-4 of it, or 2^-10 of the scale near 0.
"""
from fractions import Fraction

import numpy as np
import pytest

from oracle import fp8, linear_w4, paged, rotary
from paper_2608_11688_amd import native

pytestmark = pytest.mark.gpu

bf16 = linear_w4.bf16


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available()
    native.lib()
    return t


def i32(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def typed(torch, dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def values(rng, shape, dtype):
    v = rng.standard_normal(shape).astype(np.float32)
    return bf16(v) if dtype == "bf16" else v.astype(np.float64)


def on_gpu(torch, v, dtype, extra=0, fill=3.0):
    """Rows [T, n] with `extra` values behind each."""
    v = v.reshape(v.shape[0], -1)
    wide = torch.full((v.shape[0], v.shape[1] + extra), fill, dtype=typed(torch, dtype), device="cuda")
    wide[:, :v.shape[1]] = torch.from_numpy(np.ascontiguousarray(v)).cuda().to(typed(torch, dtype))
    return wide


def check_turned(got, want, size, dtype, unit=2.0 ** -22):
    err = np.abs(got - want)
    assert (err <= unit * size + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)).all(), err.max()


def rotation(torch, layout, dim, base=10000.0, scaling="plain", factor=1.0, amplitude=1.0):
    f = np.zeros(dim // 2)
    native.apex_rotary_frequencies(dim, base, scaling, factor, 4096.0, 1.0, 32.0, f)
    df = torch.from_numpy(f).cuda()
    return native.rotary(layout, dim, df, amplitude), f, df, np.float32(amplitude).astype(np.float64)


# T, heads, hd, dim, positions up to, extra
CASES = [(1, 1, 16, 16, 10, 0), (1, 40, 128, 128, 100000, 0), (3, 7, 64, 32, 5000, 8), (5, 3, 80, 48, 1000, 0),
         (33, 24, 128, 128, 131072, 16), (2, 9, 1024, 1024, 4000, 0), (4, 5, 1024, 16, 4000, 8), (7, 2, 256, 96, 77, 0),
         (200, 6, 64, 64, 1000000, 0), (1030, 3, 128, 64, 1 << 20, 8), (1027, 70, 16, 16, 3, 0), (2, 1, 24, 16, 9, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,heads,hd,dim,far,extra", CASES, ids=[str(c) for c in CASES])
def test_rotary(torch, T, heads, hd, dim, far, extra, layout, dtype):
    rng = np.random.default_rng(T + hd)
    x = values(rng, (T, heads, hd), dtype)
    pos = rng.integers(0, far + 1, T)
    pos[-1] = far
    pos[rng.random(T) < 0.1] = -1
    pos[0] = min(pos[0], 5) if T > 1 else far
    rot, f, keep, amplitude = rotation(torch, layout, dim, amplitude=1.19)
    dx = on_gpu(torch, x, dtype, extra)
    out = torch.full_like(dx, 7.0)
    native.apex_rotary(rot, dx, dtype, T, heads, hd, dx.stride(0), i32(torch, pos), out, out.stride(0))
    wide = out.double().cpu().numpy()
    assert (wide[:, heads * hd:] == 7).all() and (wide[pos < 0] == 7).all()
    got = wide[:, :heads * hd].reshape(T, heads, hd)
    live = pos >= 0
    want, size = rotary.turn(x[live], pos[live], f, amplitude, layout)
    check_turned(got[live], want, size, dtype)
    assert np.array_equal(got[live][..., dim:], x[live][..., dim:])
    # in place, the same bits
    native.apex_rotary(rot, dx, dtype, T, heads, hd, dx.stride(0), i32(torch, pos), dx, dx.stride(0))
    dead = torch.from_numpy(~live).cuda()
    assert torch.equal(dx[~dead, :heads * hd], out[~dead, :heads * hd])
    assert (dx[:, heads * hd:] == 3).all() and np.array_equal(
        dx[dead, :heads * hd].double().cpu().numpy(), x[~live].reshape((~live).sum(), heads * hd))


@pytest.mark.parametrize("scaling,factor", [("linear", 8.0), ("base", 4.0), ("turns", 8.0), ("index", 32.0)])
def test_scaled_frequencies(torch, scaling, factor):
    rng = np.random.default_rng(3)
    x, pos = values(rng, (6, 2, 128), "fp32"), np.array([0, 1, 4095, 4096, 100000, 131071])
    rot, f, keep, a = rotation(torch, "half", 128, 500000.0, scaling, factor)
    dx = on_gpu(torch, x, "fp32")
    native.apex_rotary(rot, dx, "fp32", 6, 2, 128, 256, i32(torch, pos), dx, 256)
    want, size = rotary.turn(x, pos, f, 1.0, "half")
    check_turned(dx.double().cpu().numpy().reshape(x.shape), want, size, "fp32")
    assert np.array_equal(dx[0].double().cpu().numpy().reshape(x.shape[1:]), x[0])      # position 0 turns nothing


def test_farthest_positions_and_turning_back(torch):
    rng = np.random.default_rng(4)
    x, pos = values(rng, (4, 3, 64), "fp32"), np.array([2 ** 31 - 1, 2 ** 31 - 2, 2 ** 30 + 1, 2 ** 24 + 1])
    rot, f, keep, a = rotation(torch, "interleaved", 64)
    dx = on_gpu(torch, x, "fp32")
    out = torch.empty_like(dx)
    native.apex_rotary(rot, dx, "fp32", 4, 3, 64, 192, i32(torch, pos), out, 192)
    want, size = rotary.turn(x, pos, f, 1.0, "interleaved")
    check_turned(out.double().cpu().numpy().reshape(x.shape), want, size, "fp32")
    minus = -keep
    back = native.rotary("interleaved", 64, minus)
    native.apex_rotary(back, out, "fp32", 4, 3, 64, 192, i32(torch, pos), out, 192)
    assert np.abs(out.double().cpu().numpy().reshape(x.shape) - x).max() <= 2.0 ** -21 * 2 * np.abs(x).max()


def test_values_that_are_not_finite_stay_in_their_pair(torch):
    x = values(np.random.default_rng(5), (2, 2, 64), "fp32")
    rot, f, keep, a = rotation(torch, "half", 32)
    clean = on_gpu(torch, x, "fp32")
    native.apex_rotary(rot, clean, "fp32", 2, 2, 64, 128, i32(torch, [9, 8]), clean, 128)
    x[1, 0, 3], x[0, 1, 40] = np.nan, np.inf          # a pair (3, 19); a value that does not turn
    dx = on_gpu(torch, x, "fp32")
    native.apex_rotary(rot, dx, "fp32", 2, 2, 64, 128, i32(torch, [9, 8]), dx, 128)
    got, want = dx.cpu().numpy().reshape(x.shape), clean.cpu().numpy().reshape(x.shape).copy()
    want[1, 0, 3] = want[1, 0, 19] = np.nan
    want[0, 1, 40] = np.inf
    assert np.array_equal(got, want, equal_nan=True)


# ------------------------------------------------------------------------------ store with rotation
class Store:
    def __init__(self, torch, T, H, G, hd, dim, layout, dtype, fmt, page, seed=0, extra=0, far=5000):
        self.torch, self.T, self.H, self.G, self.hd, self.fmt, self.dtype, self.page = torch, T, H, G, hd, fmt, dtype, page
        rng = np.random.default_rng(seed)
        self.n_pages = T // page + 3
        self.q, self.k, self.v = (values(rng, (T, n, hd), dtype) for n in (H, G, G))
        self.k *= 4.0
        self.pos = rng.integers(0, far, T)
        self.slots = rng.permutation(self.n_pages * page)[:T]
        if T > 4:
            self.pos[1], self.slots[2], self.slots[3], self.pos[4] = -1, -1, self.n_pages * page, -5
            self.v[0, 0], self.k[0, G - 1] = 0.0, 0.0
        self.layout, self.dim = layout, dim
        self.rot, self.f, self.keep, self.amplitude = rotation(torch, layout, dim, amplitude=1.1)
        # a fused projection's rows: queries, keys, values side by side
        rows = np.concatenate([x.reshape(T, -1) for x in (self.q, self.k, self.v)], 1)
        self.rows = on_gpu(torch, rows, dtype, extra)
        self.dq, self.dk, self.dv = (self.rows[:, a * hd:b * hd] for a, b in ((0, H), (H, H + G), (H + G, H + 2 * G)))
        shape = (self.n_pages, G, page, hd)
        kind = torch.bfloat16 if fmt == "bf16" else torch.uint8
        self.pools = [torch.full(shape, 9, dtype=kind, device="cuda") for _ in range(2)]
        self.scales = [None if fmt == "bf16" else torch.full(shape[:3], 9.0, device="cuda") for _ in range(2)]
        self.cache = native.paged_cache(fmt, G, hd, page, self.n_pages, *self.pools, *self.scales)
        self.q_out = torch.full((T, H * hd + 8), 7.0, dtype=typed(torch, dtype), device="cuda")
        self.dslots, self.dpos = i32(torch, self.slots), i32(torch, self.pos)

    def call(self, stream=None, q_out=None):
        out = self.q_out if q_out is None else q_out
        native.apex_paged_store_rotary(self.cache, self.rot, self.dq, self.dk, self.dv, self.dtype, self.T, self.H,
                                       self.rows.stride(0), self.rows.stride(0), self.rows.stride(0), self.dslots,
                                       self.dpos, out, out.stride(0), stream)

    def check(self):
        T, H, G, hd, page = self.T, self.H, self.G, self.hd, self.page
        live = self.pos >= 0
        wide = self.q_out.double().cpu().numpy()
        assert (wide[:, H * hd:] == 7).all() and (wide[~live] == 7).all()
        if H:
            want, size = rotary.turn(self.q[live], self.pos[live], self.f, self.amplitude, self.layout)
            check_turned(wide[live, :H * hd].reshape(-1, H, hd), want, size, self.dtype)
        kept = live & (self.slots >= 0) & (self.slots < self.n_pages * page)
        turned = rotary.turn(self.k[kept], self.pos[kept], self.f, self.amplitude, self.layout)
        plain = self.v[kept], np.zeros_like(self.v[kept])
        slots = self.slots[kept]
        for (want, size), pool, scales, exact in ((turned, *self.pool(0), False), (plain, *self.pool(1), True)):
            touched = np.zeros((self.n_pages, page), bool)
            touched[slots // page, slots % page] = True
            untouched = np.broadcast_to(~touched[:, None], pool.shape[:3])
            assert (pool[untouched] == 9).all()
            got = pool[slots // page, :, slots % page]
            if self.fmt == "bf16":
                check_turned(got, want, size, "bf16")
                if exact:
                    assert np.array_equal(got, bf16(want.astype(np.float32)))
                continue
            assert (scales[untouched] == 9).all()
            s = scales[slots // page, :, slots % page].astype(np.float64)
            peak = np.abs(want).max(-1)
            # the largest value is off by as much as any turned one
            assert (np.abs(s * 448 - peak) <= 2.0 ** -22 * size.max(-1) + 2.0 ** -23 * peak).all()
            err = np.abs(fp8.decode_array(got.astype(np.uint8)) * s[..., None] - want)
            near = 2.0 ** -22 * size + 2.0 ** -22 * np.abs(want)
            assert (err <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * s[..., None]) * (1 + 2.0 ** -10) + near).all()
            if exact:
                for i in range(len(slots)):
                    for g in range(G):
                        codes, scale = paged.quantise_row(want[i, g])
                        assert np.array_equal(got[i, g].astype(np.uint8), codes) and s[i, g] == scale

    def pool(self, i):
        p = self.pools[i].double() if self.fmt == "bf16" else self.pools[i]
        return p.cpu().numpy(), None if self.scales[i] is None else self.scales[i].cpu().numpy()


# T, H, G, hd, dim, page, extra
STORES = [(1, 1, 1, 64, 64, 16, 0), (1, 32, 8, 128, 128, 64, 0), (9, 6, 2, 64, 32, 16, 8), (33, 16, 16, 128, 48, 32, 0),
          (70, 5, 1, 64, 16, 128, 0), (40, 0, 3, 128, 128, 16, 8), (130, 24, 8, 64, 64, 1024, 8), (1030, 3, 1, 128, 96, 256, 0),
          (20, 2, 40, 64, 48, 16, 0)]
FORMATS = [(d, f) for d in ("bf16", "fp32") for f in ("bf16", "fp8")]


@pytest.mark.parametrize("dtype,fmt", FORMATS, ids=["-".join(f) for f in FORMATS])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,H,G,hd,dim,page,extra", STORES, ids=[str(c) for c in STORES])
def test_store_rotary(torch, T, H, G, hd, dim, page, extra, layout, dtype, fmt):
    c = Store(torch, T, H, G, hd, dim, layout, dtype, fmt, page, seed=T + dim, extra=extra)
    c.call()
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("dtype,fmt", [("fp32", "bf16"), ("fp32", "fp8"), ("bf16", "bf16")])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_is_rotary_then_store(torch, layout, dtype, fmt):
    """The same bits as the two calls where these round no more often; in place of the queries."""
    c = Store(torch, 50, 12, 4, 128, 64, layout, dtype, fmt, 16, seed=6)
    c.call()
    pools = [p.clone() for p in c.pools]
    scales = [s if s is None else s.clone() for s in c.scales]
    for p in c.pools:
        p.fill_(9)
    turned = c.rows.clone()
    native.apex_rotary(c.rot, c.rows, dtype, 50, 16, 128, c.rows.stride(0), c.dpos, turned, turned.stride(0))
    slots = torch.where(c.dpos >= 0, c.dslots, -1)
    native.apex_paged_store(c.cache, turned[:, 12 * 128:], turned[:, 16 * 128:], dtype, 50, turned.stride(0),
                            turned.stride(0), slots)
    assert all(torch.equal(a, b) for a, b in zip(pools, c.pools))
    assert fmt == "bf16" or all(torch.equal(a, b) for a, b in zip(scales, c.scales))
    live = c.dpos >= 0
    assert torch.equal(c.q_out[live, :12 * 128], turned[live, :12 * 128])
    c.call(q_out=c.dq)
    assert torch.equal(c.dq, torch.where(live[:, None], turned[:, :12 * 128], c.dq))


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_rows_that_are_not_finite(torch, fmt):
    c = Store(torch, 3, 2, 2, 64, 32, "half", "fp32", fmt, 16)
    c.dk[1, 5], c.dv[2, 64 + 50] = float("nan"), float("inf")
    c.call()
    torch.cuda.synchronize()
    (k, ks), (v, vs) = c.pool(0), c.pool(1)
    s = c.slots
    if fmt == "bf16":
        row = k[s[1] // 16, 0, s[1] % 16]
        assert np.isnan(row[[5, 21]]).all() and np.isfinite(np.delete(row, [5, 21])).all()
        assert np.isinf(v[s[2] // 16, 1, s[2] % 16, 50])
    else:
        assert np.isnan(ks[s[1] // 16, 0, s[1] % 16]) and np.isnan(vs[s[2] // 16, 1, s[2] % 16])
        assert np.isfinite(ks[s[1] // 16, 1, s[1] % 16]) and np.isfinite(ks[s[0] // 16, :, s[0] % 16]).all()


def test_keys_and_values_alone(torch):
    c = Store(torch, 5, 0, 2, 64, 64, "half", "bf16", "bf16", 16)
    native.apex_paged_store_rotary(c.cache, c.rot, None, c.dk, c.dv, "bf16", 5, 0, 0, c.rows.stride(0),
                                   c.rows.stride(0), c.dslots, c.dpos, None, 0)
    c.check()


def test_bits_of_values_are_kept(torch):
    """bf16 values into a bf16 pool, NaN payloads and negative zeros too, and values behind dim."""
    c = Store(torch, 2, 1, 1, 128, 32, "interleaved", "bf16", "bf16", 16, seed=3)
    bits = torch.from_numpy(np.random.default_rng(0).integers(-2 ** 15, 2 ** 15, (2, 128)).astype(np.int16)).cuda()
    bits[0, :4] = torch.tensor([0x7f81, 0x7fff, -0x8000, -0x7f], dtype=torch.int16)
    bits[:, 40] = 0x7f85
    c.dv.copy_(bits.view(torch.bfloat16))
    c.dk[:, 32:].copy_(bits[:, 32:].view(torch.bfloat16))
    c.dq[:, 32:].copy_(bits[:, 32:].view(torch.bfloat16))
    c.call()
    for t in range(2):
        page, at = int(c.slots[t]) // 16, int(c.slots[t]) % 16
        assert torch.equal(c.pools[1][page, 0, at].view(torch.int16), bits[t])
        assert torch.equal(c.pools[0][page, 0, at, 32:].view(torch.int16), bits[t, 32:])
    assert torch.equal(c.q_out[:, 32:128].view(torch.int16), bits[:, 32:])
    out = torch.empty_like(c.dq)
    native.apex_rotary(c.rot, c.dq, "bf16", 2, 1, 128, c.rows.stride(0), c.dpos, out, 128)
    assert torch.equal(out[:, 32:].contiguous().view(torch.int16), bits[:, 32:])


def test_captured_and_replayed(torch):
    c = Store(torch, 40, 8, 2, 64, 64, "half", "fp32", "fp8", 16, seed=8)
    c.call()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            c.call(stream=side.cuda_stream)
            native.apex_rotary(c.rot, c.q_out, "fp32", 40, 8, 64, c.q_out.stride(0), c.dpos, c.q_out, c.q_out.stride(0),
                               side.cuda_stream)
    for i in range(3):
        c.dpos.copy_(i32(torch, (c.pos + 17 * i) * np.where(c.pos < 0, 0, 1) - (c.pos < 0)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in (c.q_out, *c.pools, *c.scales)]
        c.call()
        native.apex_rotary(c.rot, c.q_out, "fp32", 40, 8, 64, c.q_out.stride(0), c.dpos, c.q_out, c.q_out.stride(0))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (c.q_out, *c.pools, *c.scales)))


def test_slots_past_2_gib_of_values(torch):
    """Pages behind the 2^31st byte and value, an E4M3 pool and a bf16 one."""
    for fmt in ("fp8", "bf16"):
        G, hd, page = 8, 128, 16
        n_pages = 2 ** 31 // (G * hd * page) + 5
        kind = torch.uint8 if fmt == "fp8" else torch.bfloat16
        pools = [torch.zeros((n_pages, G, page, hd), dtype=kind, device="cuda") for _ in range(2)]
        scales = [torch.zeros((n_pages, G, page), device="cuda") if fmt == "fp8" else None for _ in range(2)]
        cache = native.paged_cache(fmt, G, hd, page, n_pages, *pools, *scales)
        rot, f, keep, a = rotation(torch, "half", hd)
        x = torch.randn(2, G * hd, device="cuda")
        slots = i32(torch, [n_pages * page - 1, 3])
        pos = i32(torch, [0, 0])                     # turns nothing
        native.apex_paged_store_rotary(cache, rot, None, x, x, "fp32", 2, 0, 0, G * hd, G * hd, slots, pos, None, 0)
        for p, s in zip(pools, scales):
            for t, (pg, at) in enumerate(((n_pages - 1, page - 1), (0, 3))):
                got = p[pg, :, at].view(torch.float8_e4m3fn).float() * s[pg, :, at, None] if fmt == "fp8" else p[pg, :, at].float()
                assert torch.allclose(got, x[t].view(G, hd), rtol=2.0 ** -4, atol=0.01)
            assert int((p != 0).sum()) <= 2 * G * hd
        del pools, scales


# ------------------------------------------------------------------------------ a step's attention block
def test_attention_block_from_the_residual_stream(torch):
    """Projection, plan, store with rotation, attention, projection back with the residual: prompts, then single tokens,
    against the same in float64 (keys and values as the pool holds them)."""
    d, H, G, hd, page, R, T = 256, 8, 2, 64, 16, 3, 48
    n_pages, nb = 24, 8
    rng = np.random.default_rng(11)
    N = (H + 2 * G) * hd
    w_in, w_out = (linear_w4.bf16((rng.standard_normal(s) * s[1] ** -0.5).astype(np.float32)) for s in ((N, d), (d, H * hd)))
    packed, dense = [], []
    for w in (w_in, w_out):
        out = np.zeros(native.apex_linear_w4_bytes(*w.shape, 64), np.uint8)
        native.apex_pack_linear_w4((w.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16), *w.shape, 64, out)
        packed.append(torch.from_numpy(out).cuda())
        q, s, z = linear_w4.unpack(out, *w.shape, 64)
        g = np.arange(w.shape[1]) // 64
        dense.append(s[:, g] * (q - z[:, g]))
    rot, f, keep, a = rotation(torch, "half", hd)
    pools = [torch.zeros(n_pages, G, page, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = native.paged_cache("bf16", G, hd, page, n_pages, *pools)
    z32 = lambda *s, fill=0: torch.full(s, fill, dtype=torch.int32, device="cuda")
    cached, seq, cu, slots, pos = z32(R), z32(R), z32(R + 1), z32(T), z32(T)
    table, free = z32(R, nb, fill=-1), torch.randperm(n_pages, device="cuda", dtype=torch.int32)
    count, left = z32(1, fill=n_pages), z32(1)
    ws = torch.empty(max(native.apex_attention_paged_workspace_bytes(T, R, H, G, hd),
                         native.apex_linear_w4_workspace_bytes(T, N, d, 64, "fp32"),
                         native.apex_linear_w4_workspace_bytes(T, d, H * hd, 64, "fp32")), dtype=torch.uint8, device="cuda")
    history = [[np.zeros((0, G, hd))] * 2 for _ in range(R)]
    done = [0] * R
    for new in ([20, 7, 1], [1, 1, 1], [1, 9, 0]):
        h = torch.randn(T, d, device="cuda")
        qkv, out = torch.zeros(T, N, device="cuda"), torch.zeros(T, H * hd, device="cuda")
        y = torch.zeros(T, d, device="cuda")
        n_new = i32(torch, new)
        native.apex_linear_w4(packed[0], N, d, 64, h, "fp32", T, d, None, None, 0, qkv, "fp32", N, ws, ws.numel())
        native.apex_paged_plan(cached, n_new, R, page, n_pages, nb, T, free, count, table, seq, cu, slots, pos, left, None)
        k, v = qkv[:, H * hd:], qkv[:, (H + G) * hd:]
        native.apex_paged_store_rotary(cache, rot, qkv, k, v, "fp32", T, H, N, N, N, slots, pos, qkv, N)
        native.apex_attention_paged(cache, qkv, "fp32", T, R, H, N, cu, seq, table, nb, 0, 0, hd ** -0.5, out, H * hd, ws,
                                    ws.numel())
        native.apex_linear_w4(packed[1], d, H * hd, 64, out, "fp32", T, H * hd, None, h, d, y, "fp32", d, ws, ws.numel())
        cached.copy_(seq)
        count.copy_(left)
        x = h.double().cpu().numpy()
        rows = (x @ dense[0].T).reshape(T, H + 2 * G, hd)
        want, t = x.copy(), 0
        for r in range(R):
            at = np.arange(done[r], done[r] + new[r])
            mine = rows[t:t + new[r]]
            turned, _ = rotary.turn(mine[:, :H + G], at, f, 1.0, "half")
            for i, new_rows in enumerate((turned[:, H:], mine[:, H + G:])):
                history[r][i] = np.concatenate([history[r][i], linear_w4.bf16(new_rows.astype(np.float32))])
            for i in range(new[r]):
                a = np.zeros((H, hd))
                for head in range(H):
                    K, V = (x[:done[r] + i + 1, head // (H // G)] for x in history[r])
                    s = K @ turned[i, head] * hd ** -0.5
                    p = np.exp(s - s.max())
                    a[head] = p @ V / p.sum()
                want[t + i] += dense[1] @ a.reshape(-1)
            t += new[r]
            done[r] += new[r]
        got = y.double().cpu().numpy()
        # 32 bits throughout (1e-6), but bf16 keys and values next to a tie: one in 2^10 of them a step, 2^-7 at
        # most, away: 2^-12 together for the values, as much for the keys' scores
        assert np.linalg.norm(got[:t] - want[:t]) <= 2.0 ** -11 * np.linalg.norm(want[:t] - x[:t])
        assert np.array_equal(got[t:], x[t:])          # rows behind the last token: the residual alone
    assert seq.tolist() == done


def cosines_and_sines(pos, f):
    """Of exact products, with 2 pi to 48 digits: float64, off by its own rounding."""
    turn = 2 * Fraction("3.14159265358979323846264338327950288419716939937510")
    angle = np.array([[float(Fraction(int(p)) * Fraction(float(w)) % turn) for w in f] for p in pos])
    return np.concatenate([np.cos(angle), np.sin(angle)], 1)


@pytest.mark.parametrize("far", [1 << 20, 1 << 31])
@pytest.mark.parametrize("amplitude", [1.0, 1.35, 0.7, -3.3])
def test_sines_times_the_amplitude_are_rounded_once(torch, amplitude, far):
    """Pairs (1, 0) come out as amplitude times cosine and sine, to within half a step of fp32 of the value, which is 2^-24 and not
    2^-25 from 1 on, and 2^-36 of the amplitude, whatever the position."""
    T, dim = 200, 128
    pos = np.random.default_rng(9).integers(0, far, T)
    pos[:3] = 0, 1, far - 1
    rot, f, keep, a = rotation(torch, "half", dim, amplitude=amplitude)
    x = torch.zeros(T, dim, device="cuda")
    x[:, :dim // 2] = 1.0
    native.apex_rotary(rot, x, "fp32", T, 1, dim, dim, i32(torch, pos), x, dim)
    want = a * cosines_and_sines(pos, f)
    err = np.abs(x.double().cpu().numpy() - want)
    step = np.spacing(np.abs(want).astype(np.float32)).astype(np.float64)
    assert (err <= step / 2 + abs(a) * (2.0 ** -36 + 2.0 ** -50)).all(), ((err - step / 2) / abs(a)).max()
    if abs(amplitude) > 1:
        assert err.max() > 2.0 ** -25


def test_rows_between_others(torch):
    """Results between the rows of a call's own inputs, in the same buffer: not refused, and right."""
    T, H, hd = 5, 3, 64
    n = H * hd
    wide = torch.randn(T, 2 * n, device="cuda")
    x, out = wide[:, :n], wide[:, n:]
    rot, f, keep, a = rotation(torch, "half", hd)
    pos = i32(torch, np.arange(T) * 7)
    want = torch.empty(T, n, device="cuda")
    native.apex_rotary(rot, x, "fp32", T, H, hd, 2 * n, pos, want, n)
    before = x.clone()
    native.apex_rotary(rot, x, "fp32", T, H, hd, 2 * n, pos, out, 2 * n)
    assert torch.equal(out, want) and torch.equal(x, before)
    native.apex_rotary(rot, x[:1], "fp32", 1, H, hd, 2 * n, pos, out[:1], 4 * n)       # one row: strides do not count
    assert torch.equal(out, want)
    with pytest.raises(native.ApexError):
        native.apex_rotary(rot, x, "fp32", T, H, hd, 2 * n, pos, wide[:, 4:], 2 * n)
