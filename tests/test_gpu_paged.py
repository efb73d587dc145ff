"""Paged-cache operators against the float64 oracle.

Attention tolerances.  Per output, with size = sum of weight * |value| and peak = the largest sum of
|scale q k| of a visible position: a score is off by at most (hd + 8) roundings of 2^-24 of its
peak, a weight by twice that (numerator and normaliser) and 32-bit sums by less than 2^-16 of `size`
(64 positions at a time, the rest in tree order over wavefronts and splits).  bf16 adds half a step,
2^-8, of every weight (of `size`) and of the output.  That bound is for each output.  Roundings
are independent, so that over all outputs the 2-norm of the error is much smaller: 2e-6 of the
result's with fp32, where a dropped 8-bit piece of an operand would leave 4e-6 and more, and with
bf16 two roundings of rms 2^-8 / sqrt(3) * 0.72 = 1.6e-3 each, 2.3e-3 together, at most 4e-3.
"""
import os
import re

import numpy as np
import pytest

from oracle import fp8
from oracle import paged as opaged
from oracle.attention import round_bf16
from paper_2608_11688_amd import native

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available()
    native.lib()
    return t


def i32(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def cdiv(a, b):
    return -(-a // b)


class Case:
    """Requests of given total and new lengths over a pool of scattered pages."""

    def __init__(self, torch, lens, new, H, G, hd, page, fmt, dtype, pad=0, seed=0, extra_q=0):
        self.torch, self.H, self.G, self.hd, self.page, self.fmt, self.dtype = torch, H, G, hd, page, fmt, dtype
        rng = np.random.default_rng(seed)
        self.rng, self.R = rng, len(lens)
        self.lens, self.new = np.array(lens), np.array(new)
        self.cu = np.concatenate([[0], np.cumsum(new)])
        self.T = int(self.cu[-1]) + pad
        blocks = [cdiv(n, page) for n in lens]
        self.n_pages, self.nb = sum(blocks) + 3, max(blocks + [1]) + 1
        order = rng.permutation(self.n_pages)
        self.table, at = np.full((self.R, self.nb), -1), 0
        for r, b in enumerate(blocks):
            self.table[r, :b] = order[at:at + b]
            at += b
        shape = (self.n_pages, G, page, hd)
        self.k, self.v = rng.standard_normal((2,) + shape)
        self.ks = self.vs = None
        if fmt == "bf16":
            self.k, self.v = round_bf16(self.k), round_bf16(self.v)
        else:
            self.ks, self.vs = (rng.random((2,) + shape[:3]) * 0.01 + 0.005).astype(np.float32)
            self.k, self.v = fp8.encode(self.k * 100), fp8.encode(self.v * 100)
        q = 2 * rng.standard_normal((self.T, H, hd))
        self.q = round_bf16(q) if dtype == "bf16" else q.astype(np.float32).astype(np.float64)
        self.extra_q = extra_q

    def type(self):
        return self.torch.bfloat16 if self.dtype == "bf16" else self.torch.float32

    def pool(self, x):
        t = self.torch.from_numpy(np.ascontiguousarray(x))
        return t.cuda() if self.fmt == "fp8" else t.cuda().to(self.torch.bfloat16)

    def values(self):
        if self.fmt == "bf16":
            return self.k, self.v
        return (fp8.decode_array(self.k) * self.ks[..., None].astype(np.float64),
                fp8.decode_array(self.v) * self.vs[..., None].astype(np.float64))

    def device(self):
        torch = self.torch
        f = lambda s: None if s is None else torch.from_numpy(s).cuda()
        self.dk, self.dv, self.dks, self.dvs = self.pool(self.k), self.pool(self.v), f(self.ks), f(self.vs)
        self.cache = native.paged_cache(self.fmt, self.G, self.hd, self.page, self.n_pages, self.dk, self.dv,
                                        self.dks, self.dvs)
        wide = torch.full((self.T, self.H * self.hd + self.extra_q), 3.0, dtype=self.type(), device="cuda")
        wide[:, :self.H * self.hd] = torch.from_numpy(self.q.reshape(self.T, -1)).cuda().to(self.type())
        self.dq = wide[:, :self.H * self.hd]
        self.out = torch.full((self.T, self.H * self.hd + self.extra_q), 7.0, dtype=self.type(), device="cuda")
        self.dcu, self.dseq, self.dtable = (i32(torch, x) for x in (self.cu, self.lens, self.table))
        n = native.apex_attention_paged_workspace_bytes(self.T, self.R, self.H, self.G, self.hd)
        self.ws = torch.full((n,), 0xAB, dtype=torch.uint8, device="cuda")

    def call(self, window=0, sinks=0, scale=None, stream=None, out=None):
        out = self.out if out is None else out
        native.apex_attention_paged(self.cache, self.dq, self.dtype, self.T, self.R, self.H, self.dq.stride(0),
                                    self.dcu, self.dseq, self.dtable, self.nb, window, sinks,
                                    scale or self.hd ** -0.5, out, out.stride(0), self.ws, self.ws.numel(), stream)

    def check(self, window=0, sinks=0, norm=True):
        self.device()
        self.call(window, sinks)
        self.torch.cuda.synchronize()
        wide = self.out.double().cpu().numpy()
        assert (wide[:, self.H * self.hd:] == 7).all()                 # between the rows
        got = wide[:, :self.H * self.hd].reshape(self.T, self.H, self.hd)
        k, v = self.values()
        with np.errstate(invalid="ignore", over="ignore"):
            want, size, peak = opaged.attend(self.q, k, v, self.cu, self.lens, self.table, window, sinks,
                                             self.hd ** -0.5, np.full_like(got, 7.0))
        return compare(got, want, size, peak, self.hd, self.dtype, norm)


def compare(got, want, size, peak, hd, dtype, norm=True):
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    step = 2.0 ** -8 if dtype == "bf16" else 0.0
    bound = size * (2 * (hd + 8) * 2.0 ** -24 * peak[..., None] + 2.0 ** -16 + step) + np.abs(want) * (step + 2.0 ** -22)
    err = np.abs(got - want)
    assert (err[ok] <= bound[ok] + 1e-30).all(), (err[ok] - bound[ok]).max()
    rel = np.linalg.norm(err[ok]) / max(np.linalg.norm(want[ok]), 1e-30)
    if norm:
        assert rel <= (4e-3 if dtype == "bf16" else 2e-6), rel
    return rel


FORMATS = [("bf16", "bf16"), ("fp8", "bf16"), ("bf16", "fp32"), ("fp8", "fp32")]
FMT_IDS = ["-".join(f) for f in FORMATS]

# single tokens: total lengths of the requests, H, G, hd, page, window, sinks
TOKENS = [
    ([1], 1, 1, 64, 16, 0, 0),                       # nothing cached but its own position
    ([2, 17, 16, 33], 6, 2, 128, 16, 0, 0),          # ends at, before and behind a page's end
    ([129, 127, 500], 8, 8, 64, 32, 0, 0),           # one query head per group
    ([300, 1, 700, 64], 20, 4, 128, 64, 0, 0),       # five heads per group
    ([1500], 7, 1, 64, 1024, 0, 0),                  # seven, one long page
    ([2100, 900], 16, 1, 128, 128, 0, 0),            # sixteen
    ([400, 90, 10], 8, 2, 128, 16, 50, 4),           # window with sinks, contexts under and over it
    ([400, 90, 10], 8, 2, 64, 32, 1, 0),             # a window of the token itself
    ([400, 300], 8, 2, 64, 16, 37, 130),             # sinks past a unit
    ([200, 60], 4, 1, 128, 16, 150, 100),            # sinks that reach into the window
    ([777], 6, 2, 128, 256, 256, 1),
]


@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
@pytest.mark.parametrize("lens,H,G,hd,page,window,sinks", TOKENS, ids=[str(c) for c in TOKENS])
def test_single_tokens(torch, lens, H, G, hd, page, window, sinks, fmt, dtype):
    c = Case(torch, lens, [1] * len(lens), H, G, hd, page, fmt, dtype, seed=1)
    print(c.check(window, sinks))


# chunks: (total, new) of the requests, H, G, hd, page, window, sinks, rows behind the last
CHUNKS = [
    ([(2, 2)], 1, 1, 64, 16, 0, 0, 0),
    ([(5, 3), (40, 7)], 4, 2, 128, 16, 0, 0, 2),
    ([(130, 130)], 4, 1, 64, 16, 0, 0, 0),                       # a whole prompt
    ([(64, 64), (65, 33), (129, 128)], 2, 2, 128, 64, 0, 0, 0),  # at the units' edges
    ([(300, 77), (1, 1), (90, 0), (200, 12)], 10, 2, 64, 32, 0, 0, 5),   # single, none, chunks; five heads
    ([(333, 100)], 16, 1, 128, 128, 0, 0, 0),                    # eight tokens a tile
    ([(300, 200)], 7, 1, 64, 16, 0, 0, 1),                       # 18 tokens and two empty rows a tile
    ([(260, 150), (70, 70)], 4, 1, 128, 16, 40, 5, 0),           # window inside a tile, sinks
    ([(500, 30), (33, 9)], 6, 2, 64, 32, 7, 0, 3),
    ([(400, 64)], 4, 2, 128, 256, 100, 70, 0),                   # sinks past a unit
    ([(1200, 6)], 2, 1, 64, 16, 0, 0, 0),                        # few rows, many units: split
    ([(700, 600)], 1, 1, 128, 512, 0, 0, 0),
]


@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
@pytest.mark.parametrize("reqs,H,G,hd,page,window,sinks,pad", CHUNKS, ids=[str(c) for c in CHUNKS])
def test_chunks(torch, reqs, H, G, hd, page, window, sinks, pad, fmt, dtype):
    c = Case(torch, [r[0] for r in reqs], [r[1] for r in reqs], H, G, hd, page, fmt, dtype, pad=pad, seed=2,
             extra_q=8 * pad)
    print(c.check(window, sinks))


# more than the 512 tiles of a launch, groups that do not divide the workgroups, one request's
# tokens among requests without any: requests, new tokens of a request, longest, H, G, hd
MANY = [
    (700, lambda rng, R: np.ones(R, int), 90, 4, 2, 64),
    (1100, lambda rng, R: rng.integers(0, 2, R), 70, 2, 1, 128),
    (600, lambda rng, R: rng.integers(8, 10, R), 40, 16, 1, 64),        # 8 tokens a tile: a second tile of one
    (40, lambda rng, R: np.where(np.arange(R) == 17, 30, 0), 300, 6, 3, 128),
    (3, lambda rng, R: np.ones(R, int), 500, 66, 33, 64),
    (2, lambda rng, R: np.ones(R, int), 600, 520, 520, 64),             # fewer workgroups than groups
    (2, lambda rng, R: np.array([70, 3]), 100, 300, 300, 64),
    (1, lambda rng, R: np.ones(R, int), 40000, 8, 1, 128),              # one tile in very many parts
]


@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
@pytest.mark.parametrize("R,new,longest,H,G,hd", MANY, ids=[f"R{c[0]}-{c[2]}-H{c[3]}-G{c[4]}" for c in MANY])
def test_many_tiles_groups_and_parts(torch, R, new, longest, H, G, hd, fmt, dtype):
    rng = np.random.default_rng(R)
    n = new(rng, R)
    lens = [longest if r == 0 else int(x + rng.integers(0, max(longest - x, 1))) for r, x in enumerate(n)]
    c = Case(torch, lens, n, H, G, hd, 16, fmt, dtype, pad=1 if R > 1 else 0, seed=12)
    print(c.check())


def one_by_one(c):
    """Whether the call's last launch took its tokens one by one (the workspace's second word)."""
    return bool(c.ws[4:8].view(c.torch.int32)[0])


@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
@pytest.mark.parametrize("R,new,longest,H,G,hd", MANY, ids=[f"R{c[0]}-{c[2]}-H{c[3]}-G{c[4]}" for c in MANY])
def test_many_tiles_groups_and_parts_without_padding(torch, R, new, longest, H, G, hd, fmt, dtype):
    rng = np.random.default_rng(R)
    n = new(rng, R)
    lens = [longest if r == 0 else int(x + rng.integers(0, max(longest - x, 1))) for r, x in enumerate(n)]
    c = Case(torch, lens, n, H, G, hd, 16, fmt, dtype, seed=12)
    c.check()
    assert one_by_one(c) == (max(n) == 1)


# Requests of few tokens among idle ones: (requests, new tokens of the first `some`, some, longest), H,
# G, hd, one by one.  The rule's two limits, on either side: tokens as many as requests, contexts
# read twice; and more tiles than workgroups.
FEW = [
    ((40, 2, 20, 300), 8, 2, 128, True), ((39, 2, 20, 300), 8, 2, 128, False),
    ((40, 3, 10, 300), 8, 2, 128, False), ((300, 3, 100, 90), 32, 16, 128, False),
    ((300, 3, 100, 90), 32, 16, 64, False), ((1600, 3, 530, 40), 4, 2, 64, False),
]


@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
@pytest.mark.parametrize("requests,H,G,hd,kind", FEW, ids=[str(c[0]) + f"-{c[3]}" for c in FEW])
def test_requests_of_few_tokens_among_idle_ones(torch, requests, H, G, hd, kind, fmt, dtype):
    R, new, some, longest = requests
    rng = np.random.default_rng(R)
    n = np.where(rng.permutation(R) < some, new, 0)
    lens = [longest if x else 0 for x in n]
    c = Case(torch, lens, n, H, G, hd, 16, fmt, dtype, seed=24, pad=R - new * some if R > new * some else 0)
    c.check()
    assert one_by_one(c) == kind


@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4)])
def test_rows_without_a_token_change_no_bit(torch, window, sinks, fmt, dtype):
    """Single tokens and a chunk with and without empty rows behind them (and, not to the bit, among
    requests that bring nothing)."""
    for lens, new in (([3000, 90, 1, 400], [1] * 4), ([900], [70])):
        c = Case(torch, lens, new, 8, 2, 128, 16, fmt, dtype, seed=25)
        c.check(window, sinks)
        first = c
        for pad, idle in ((1, 0), (50, 0), (0, 90), (7, 3)):
            c = Case(torch, lens + [0] * idle, new + [0] * idle, 8, 2, 128, 16, fmt, dtype, pad=pad, seed=25)
            assert c.n_pages == first.n_pages and c.cu[len(new)] == len(first.q)
            c.k, c.v, c.ks, c.vs = first.k, first.v, first.ks, first.vs
            c.q[:len(first.q)], c.table[:len(lens)] = first.q, first.table
            c.check(window, sinks)
            assert one_by_one(c) == (new[0] == 1)
            assert idle or torch.equal(c.out[:len(first.q)], first.out), (pad, idle)


@pytest.mark.parametrize("spread", [0.0, 3.0])
@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_padded_single_tokens_have_weights_of_16_bits(torch, fmt, spread):
    """As test_weights_are_held_to_more_bits_than_the_result, whose bound this is, with empty rows."""
    for seed in range(4):
        c = Case(torch, [2, 5, 31], [1] * 3, 8, 2, 128, 16, fmt, "bf16", pad=30, seed=60 + seed)
        if c.vs is not None:
            c.vs *= np.exp(c.rng.uniform(-spread, spread, c.vs.shape)).astype(np.float32)
        c.check()
        k, v = c.values()
        want = opaged.attend(c.q, k, v, c.cu, c.lens, c.table, 0, 0, 128 ** -0.5, np.zeros((c.T, 8, 128)))[0][:3]
        got = c.out.double().cpu().numpy().reshape(c.T, 8, 128)[:3]
        assert np.linalg.norm(got - want) <= 1.05 * np.linalg.norm(round_bf16(want) - want)


def test_a_captured_call_serves_any_lengths(torch):
    """One graph over 24 rows and 24 requests: single tokens, a chunk, both, none, replayed in turn."""
    c = Case(torch, [400] * 24, [1] * 24, 8, 2, 128, 16, "fp8", "bf16", seed=26)
    c.device()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.call(stream=torch.cuda.current_stream().cuda_stream)
    k, v = c.values()
    for new in ([1] * 24, [0] * 5 + [24] + [0] * 18, [1] * 8 + [9] + [0] * 8 + [1] * 7, [1] * 4 + [16] + [0] * 19, [0] * 24,
                [2] * 12 + [0] * 12, [1] * 24):
        cu = np.concatenate([[0], np.cumsum(new)])
        lens = c.rng.integers(24, 401, 24)
        c.dcu.copy_(i32(torch, cu)), c.dseq.copy_(i32(torch, lens))
        c.out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = c.out.double().cpu().numpy().reshape(24, 8, 128)
        want, size, peak = opaged.attend(c.q, k, v, cu, lens, c.table, 0, 0, 128 ** -0.5, np.full_like(got, 7.0))
        compare(got, want, size, peak, 128, "bf16")
        new = np.array(new)
        assert one_by_one(c) == ((new * lens).sum() <= 2 * lens[new > 0].sum())


@pytest.mark.parametrize("new", [1, 90])
def test_as_many_rows_as_there_may_be(torch, new):
    """All but a few of 2^20 rows empty: the launches behind the first find no tile."""
    c = Case(torch, [500, 40, 300], [new, 1, new], 2, 1, 64, 16, "bf16", "bf16", seed=29)
    c.check()
    want = c.out.clone()
    live, c.T = c.T, native.MAX_STEP_TOKENS
    wide = torch.full((c.T, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    wide[:live] = c.dq
    c.dq, c.out = wide, torch.full_like(wide, 7.0)
    c.ws = torch.full((native.apex_attention_paged_workspace_bytes(c.T, c.R, 2, 1, 64),), 0xAB, dtype=torch.uint8,
                      device="cuda")
    c.call()
    assert torch.equal(c.out[:live], want) and (c.out[live:] == 7).all()


@pytest.mark.parametrize("pad", [0, 3])
def test_as_many_single_tokens_as_there_may_be(torch, pad):
    """4096 requests of one token each, eight launches over one workspace; a sample against the oracle."""
    rng = np.random.default_rng(27)
    n = rng.integers(1, 41, native.MAX_REQUESTS)
    c = Case(torch, n, [1] * len(n), 16, 2, 64, 16, "bf16", "bf16", pad=pad, seed=27)
    c.device()
    c.call()
    got = c.out.double().cpu().numpy().reshape(c.T, 16, 64)
    assert one_by_one(c) and (got[len(n):] == 7).all()
    for r in [0, 1, 511, 512, *rng.integers(0, len(n), 40), len(n) - 1]:
        want, size, peak = opaged.attend(c.q[r:r + 1], c.k, c.v, [0, 1], n[r:r + 1], c.table[r:r + 1], 0, 0, 0.125,
                                         np.zeros((1, 16, 64)))
        compare(got[r:r + 1], want, size, peak, 64, "bf16", norm=False)


@pytest.mark.parametrize("fmt,new,pad", [("bf16", 1, 0), ("fp8", 1, 0), ("fp8", 1, 9), ("fp8", 30, 0)])
@pytest.mark.parametrize("spread", [0.0, 3.0])
def test_weights_are_held_to_more_bits_than_the_result(torch, fmt, new, pad, spread):
    """16 bits (single tokens) or fp16's 11 of weight times scale (E4M3): in the 2-norm at most an
    eighth of what rounding the result to bf16 gives, 1.008 times that together, and 1.05 with the
    chance that the few hundred outputs here leave.  Few positions, so that single weights tell, and
    scales e^spread apart."""
    for seed in range(4):
        c = Case(torch, [new + 1, new + 4, new + 30], [new] * 3, 8, 2, 128, 16, fmt, "bf16", pad=pad, seed=40 + seed)
        if c.vs is not None:
            c.vs *= np.exp(c.rng.uniform(-spread, spread, c.vs.shape)).astype(np.float32)
        c.check()
        n = 3 * new
        k, v = c.values()
        want = opaged.attend(c.q, k, v, c.cu, c.lens, c.table, 0, 0, 128 ** -0.5, np.zeros((c.T, 8, 128)))[0][:n]
        got = c.out.double().cpu().numpy().reshape(c.T, 8, 128)[:n]
        assert np.linalg.norm(got - want) <= 1.05 * np.linalg.norm(round_bf16(want) - want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("factor", [1e-28, 1e28])
def test_scales_far_from_one(torch, factor, new, dtype):
    """All of a pool's values tiny or huge, and zero rows among them."""
    c = Case(torch, [90, 200], [new, new], 4, 2, 64, 16, "fp8", dtype, pad=new > 1, seed=14)
    c.vs *= np.float32(factor)
    c.vs[c.rng.random(c.vs.shape) < 0.1] = 0
    c.check()


@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("gap", [8, 25.2, 33, 60, 90])
def test_small_weights_beside_a_very_large_one(torch, gap, new, fmt, dtype):
    """The first position's weight stands `gap` powers of two above those of all others, and half of
    its values are 0: these outputs are made up by the others and held to the same bound."""
    c = Case(torch, [300, 150], [new, new], 4, 2, 64, 16, fmt, dtype, seed=18)
    encode = fp8.encode if fmt == "fp8" else round_bf16
    c.q[:], c.q[..., 0] = 0, gap * np.log(2)
    c.q = round_bf16(c.q) if dtype == "bf16" else c.q.astype(np.float32).astype(np.float64)
    c.k[..., 0] = encode(np.zeros(c.k.shape[:3]))
    first = c.table[:2, 0]
    c.k[first, :, 0, 0] = encode(np.full((2, 2), 8.0))       # scale 1/8: a score of gap * ln 2
    c.v[first, :, 0, 32:] = encode(np.zeros((2, 2, 32)))
    if c.ks is not None:
        c.ks[first, :, 0] = 1.0
    c.check()
    assert (c.out.view(c.T, 4, 64)[:, :, 32:] != 0).float().mean() > 0.9


@pytest.mark.parametrize("power,dtype", [(-100, "bf16"), (112, "bf16"), (112, "fp32")])
@pytest.mark.parametrize("new", [1, 40])
def test_scales_as_far_from_one_as_values_go(torch, power, new, dtype):
    """All value scales of a request near the ends of the type's range, zeros among them.  Pieces of
    weight times scale below 2^-126 may be lost: with scales of 2^-107 the second pieces of weights
    under 2^-11, 2^-18 of a weight of 1 each, where the bound has 2^-8 of all weights."""
    c = Case(torch, [90, 200], [new, new], 4, 2, 64, 16, "fp8", dtype, pad=new > 1, seed=19)
    c.vs *= np.float32(2.0 ** power)
    c.vs[c.rng.random(c.vs.shape) < 0.1] = 0
    c.device()
    c.call()
    k, v = c.values()
    got = c.out.double().cpu().numpy().reshape(c.T, 4, 64)
    rows = slice(0, 2 * new)
    want, size, peak = opaged.attend(c.q, k, v, c.cu, c.lens, c.table, 0, 0, 0.125, np.zeros_like(got))
    up = 2.0 ** -power
    compare(got[rows] * up, want[rows] * up, size[rows] * up, peak[rows], 64, dtype)


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_as_many_requests_as_there_may_be(torch, fmt):
    """4096 prompts of 1 to 40 tokens, ten launches; a sample of them against the oracle."""
    rng = np.random.default_rng(15)
    n = rng.integers(1, 41, native.MAX_REQUESTS)
    c = Case(torch, n, n, 16, 2, 64, 16, fmt, "bf16", pad=3, seed=15)
    c.device()
    c.call()
    got = c.out.double().cpu().numpy().reshape(c.T, 16, 64)
    assert (got[-3:] == 7).all()
    k, v = c.values()
    for r in [0, 1, *rng.integers(0, len(n), 40), len(n) - 1]:
        rows = slice(c.cu[r], c.cu[r + 1])
        want, size, peak = opaged.attend(c.q[rows], k, v, [0, n[r]], n[r:r + 1], c.table[r:r + 1], 0, 0, 0.125,
                                         np.zeros((n[r], 16, 64)))
        compare(got[rows], want, size, peak, 64, "bf16", norm=False)


@pytest.mark.parametrize("H", [1, 16])
def test_lengths_that_count_tokens_twice_stay_inside(torch, H):
    """cu_new that goes back and forth: more tiles than T tokens have.  Which rows are written is
    open; nothing outside of `out` and the workspace is."""
    c = Case(torch, [40] * 6, [4] * 6, H, 1, 64, 16, "bf16", "bf16", seed=13)
    c.device()
    n = c.ws.numel()
    c.ws = torch.full((n + 65536,), 0xAB, dtype=torch.uint8, device="cuda")
    c.dcu.copy_(i32(torch, [0, 24, 0, 24, 0, 24, 0]))
    native.apex_attention_paged(c.cache, c.dq, "bf16", c.T, c.R, H, c.dq.stride(0), c.dcu, c.dseq, c.dtable, c.nb, 0,
                                0, 0.125, c.out, c.out.stride(0), c.ws, n)
    torch.cuda.synchronize()
    assert (c.ws[n:] == 0xAB).all()


@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
@pytest.mark.parametrize("new", [1, 6])
def test_pages_with_ids_out_of_range_are_left_out(torch, new, fmt, dtype):
    c = Case(torch, [200, 150, 40], [new] * 3, 4, 2, 64, 16, fmt, dtype, seed=3)
    c.table[0, [0, 5, 12]] = [-1, c.n_pages, 2 ** 31 - 1]   # the first, an inner one, its last
    c.table[1, 3] = -2 ** 31
    c.table[2, :] = -7                                       # sees nothing: zeros
    c.check()
    assert (c.out[2 * new:] == 0).all()


@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
@pytest.mark.parametrize("new,window,sinks", [(1, 0, 0), (1, 20, 3), (9, 0, 0), (9, 20, 3), (70, 33, 5)])
def test_what_a_row_does_not_see_does_not_reach_it(torch, new, window, sinks, fmt, dtype):
    """NaN and infinities behind the last position, under the window, in the first positions'
    shadow and at later tokens of the same chunk."""
    c = Case(torch, [150, 37 + new], [new, new], 4, 2, 128, 16, fmt, dtype, seed=4)
    bad = np.float32("nan")

    def spoil(pid, off):
        if fmt == "fp8":
            c.v[pid, :, off, 5], c.k[pid, :, off, 9] = 0x7F, 0xFF
            c.vs[pid, :, off] = c.ks[pid, :, off] = bad if off % 2 else np.inf
        else:
            c.v[pid, :, off, 5], c.v[pid, :, off, 70], c.k[pid, :, off, 9] = np.inf, bad, -np.inf

    for r in range(2):
        n = int(c.lens[r])
        last = n - (new + 1) // 2 if new > 1 else n              # from here on only later tokens see it
        first = n - new
        for j in range(c.nb * 16):
            pid = c.table[r, j // 16]
            if pid >= 0 and (j >= last or (window and sinks <= j <= first - window)):
                spoil(pid, j % 16)
    free = sorted(set(range(c.n_pages)) - set(c.table.ravel()))
    for pid in free:
        for off in range(16):
            spoil(pid, off)
    # rows that see a spoiled position are NaN (or infinite) by their own right: not compared
    k, v = c.values()
    c.device()
    c.call(window, sinks)
    torch.cuda.synchronize()
    got = c.out.double().cpu().numpy().reshape(c.T, 4, 128)
    with np.errstate(invalid="ignore", over="ignore"):
        want, size, peak = opaged.attend(c.q, k, v, c.cu, c.lens, c.table, window, sinks, 128 ** -0.5, got)
    clean = np.isfinite(size).all(axis=(1, 2)) & np.isfinite(peak).all(axis=1)
    assert clean.sum() >= 2 * (new // 2 if new > 1 else 1)
    compare(got[clean], want[clean], size[clean], peak[clean], 128, dtype)
    if new > 1:
        assert not np.isfinite(got[~clean]).all()


@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
@pytest.mark.parametrize("new", [1, 70])
def test_table_entries_that_no_row_sees_have_no_effect(torch, new, fmt, dtype):
    """Past the last position and under the window: any numbers, page ids of other requests among
    them."""
    c = Case(torch, [900, 333 + new], [new, new], 4, 2, 64, 16, fmt, dtype, seed=28)
    c.check(100, 20)
    want = c.out.clone()
    table = c.table.copy()
    for r in range(2):
        n, first = int(c.lens[r]), int(c.lens[r]) - new
        for b in range(c.nb):
            if b * 16 >= n or (b * 16 >= 20 and b * 16 + 15 <= first - 100):
                table[r, b] = c.rng.choice([-1, 2 ** 31 - 1, -2 ** 31, c.n_pages, *c.table[1 - r][:9]])
    assert (table != c.table).sum() > 30
    c.dtable.copy_(i32(torch, table))
    c.out.fill_(7.0)
    c.call(100, 20)
    assert torch.equal(c.out, want)


def test_a_nan_that_is_seen_is_nan(torch):
    c = Case(torch, [50], [1], 2, 1, 64, 16, "bf16", "bf16", seed=5)
    c.v[c.table[0, 1], 0, 3, 7] = np.nan
    c.device()
    c.call()
    got = c.out.view(2, 64)
    assert torch.isnan(got[:, 7]).all() and torch.isnan(got).sum() == 2


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new,pad", [(1, 0), (1, 1), (40, 0)])
def test_keys_of_minus_infinity_have_no_weight(torch, new, pad, dtype):
    """Scores of -infinity are weights of 0, and rows that have no others are 0: the queries are bf16
    numbers, so that an fp32 one is all in its first piece."""
    c = Case(torch, [150, 90, 200], [new, new, new], 4, 2, 64, 16, "bf16", dtype, pad=pad, seed=20)
    c.q = round_bf16(c.q)
    c.q[..., 3] = np.abs(c.q[..., 3]) + 1
    c.q[1, :, 11] = 1.0 + 2.0 ** -7
    gone = c.rng.random(c.k.shape[:3]) < 0.3
    gone[c.table[1, :cdiv(90, 16)]] = True                  # all of the second request's
    gone[c.table[2, 12], :, 7] = False                      # the third's last is there
    k, v = c.k.copy(), c.v
    c.k[gone, 3] = -np.inf
    c.device()
    c.call()
    got = c.out.double().cpu().numpy().reshape(c.T, 4, 64)
    keys = k.copy()
    keys[gone, 3] = -1e9                                    # weights of 0 in 64 bits as well
    want, size, _ = opaged.attend(c.q, keys, v, c.cu, c.lens, c.table, 0, 0, 0.125, np.full_like(got, 7.0))
    keys[gone, 3] = 0
    peak = opaged.attend(c.q, keys, v, c.cu, c.lens, c.table, 0, 0, 0.125, np.full_like(got, 7.0))[2]
    rows = slice(new, 2 * new)
    assert (got[rows] == 0).all()
    want[rows] = size[rows] = 0
    compare(got, want, size, peak, 64, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new,pad", [(1, 0), (1, 1), (40, 0)])
def test_queries_that_are_infinite(torch, new, pad, dtype):
    """-infinity against keys of one sign: all scores -infinity, zeros; +infinity: NaN."""
    c = Case(torch, [50, 70], [new, new], 2, 1, 64, 16, "bf16", dtype, pad=pad, seed=21)
    c.k[..., 9] = np.abs(c.k[..., 9]) + 0.5
    c.q[:, 0, 9], c.q[:, 1, 9] = -np.inf, np.inf
    c.device()
    c.call()
    got = c.out.view(c.T, 2, 64)[:2 * new]
    assert (got[:, 0] == 0).all() and torch.isnan(got[:, 1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new,pad", [(1, 0), (1, 1), (40, 0)])
def test_values_that_are_infinite_and_seen(torch, new, pad, dtype):
    """A weight times an infinite value is that infinity, whatever pieces the weight is held in; of
    weight 1 (one position), and among others."""
    c = Case(torch, [new, 90 + new, 300], [new, new, new], 4, 2, 64, 16, "bf16", dtype, pad=pad, seed=22)
    c.v[c.table[:, 0], :, 0, 5:8] = np.inf, -np.inf, np.nan
    c.v[c.table[2, 17], :, 0, 5] = -np.inf                  # with another sign: NaN
    c.device()
    c.call()
    got = c.out.double().cpu().numpy().reshape(c.T, 4, 64)
    with np.errstate(invalid="ignore"):
        want, size, peak = opaged.attend(c.q, c.k, c.v, c.cu, c.lens, c.table, 0, 0, 0.125, np.full_like(got, 7.0))
    assert np.isinf(want).any() and np.array_equal(np.isinf(got), np.isinf(want))
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    infinite = np.isinf(want)
    for x in (got, want, size):
        x[infinite] = 0
    compare(got, want, size, peak, 64, dtype)


@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 3)])
@pytest.mark.parametrize("new,pad", [(1, 0), (1, 1), (90, 0)])
def test_weights_of_zero_meet_values_that_are_not_finite(torch, new, pad, window, sinks, fmt, dtype):
    """Seen values that are no finite numbers, with weights that are 0 in 32 bits: NaN or infinite for
    each row that sees them, also where other rows of a tile do not, and nothing for those."""
    c = Case(torch, [new + 200, new + 37, new], [new] * 3, 4, 2, 64, 16, fmt, dtype, pad=pad, seed=23)
    encode = fp8.encode if fmt == "fp8" else round_bf16
    c.q[..., 0] = 64.0
    c.k[..., 0] = encode(np.ones(c.k.shape[:3]) * 8)
    if c.ks is not None:
        c.ks[:] = 1 / 8
        c.k[..., 1:] = encode(c.rng.standard_normal(c.k.shape[:3] + (63,)) * 8)
    spoilt = []                                             # a position of each page of each request
    for r in range(3):
        for j in range(5, int(c.lens[r]), 16):
            pid = c.table[r, j // 16]
            c.k[pid, :, j % 16, 0] = encode(np.full(2, -256.0))     # scores of -256 and less
            c.v[pid, :, j % 16, 9] = np.inf if fmt == "bf16" else 0x7F
            spoilt.append((r, j))
    v = c.v.copy()
    c.device()
    c.call(window, sinks)
    got = c.out.double().cpu().numpy().reshape(c.T, 4, 64)
    for r, j in spoilt:
        v[c.table[r, j // 16], :, j % 16, 9] = 0
    c.v = v
    want, size, peak = opaged.attend(c.q, *c.values(), c.cu, c.lens, c.table, window, sinks, 0.125, np.full_like(got, 7.0))
    sees = np.zeros(c.T, bool)
    for r in range(3):
        for i in range(new):
            seen = opaged.visible_positions(int(c.lens[r]) - new + i, window, sinks)
            sees[c.cu[r] + i] = (seen % 16 == 5).any()
    assert not np.isfinite(got[sees][..., 9]).any()
    got[sees, :, 9] = want[sees, :, 9]
    compare(got, want, size, peak, 64, dtype, norm=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 40])
def test_large_and_even_scores(torch, new, dtype):
    """Scores that stand far apart (weights of one position only) and all equal ones."""
    c = Case(torch, [333], [new], 4, 2, 64, 16, "bf16", dtype, seed=6)
    c.q = round_bf16(c.q * 64)
    c.check(norm=False)
    c.q[:] = 0
    c.check()


def test_lengths_that_disagree_stay_inside(torch):
    """Lengths shorter than the new tokens, past the table, no ascending list: zeros or clamped, no
    access out of range (positions a token would have before 0 see nothing)."""
    c = Case(torch, [40, 64, 48], [4, 2, 3], 2, 1, 64, 16, "bf16", "bf16", seed=7)
    c.device()
    c.dseq.copy_(i32(torch, [2, 10 ** 9, -5]))
    c.call()
    torch.cuda.synchronize()
    assert (c.out[:2] == 0).all() and (c.out[2:4] != 0).any(dim=1).all()
    assert (c.out[6:9] == 0).all()
    c.dcu.copy_(i32(torch, [-3, 10 ** 9, 2, -1]))
    c.call()
    torch.cuda.synchronize()


@pytest.mark.parametrize("new", [1, 70])
def test_windows_and_sinks_as_large_as_they_may_be(torch, new):
    """As none: the same positions, the same bits."""
    big = 2 ** 31 - 1
    c = Case(torch, [300, 90], [new, new], 4, 2, 64, 16, "bf16", "bf16", pad=2, seed=16)
    c.check()
    want = c.out.clone()
    for window, sinks in ((big, 0), (big, big), (1, big), (0, big), (200, 200)):
        c.out.fill_(7.0)
        c.call(window, sinks)
        if window == 200:
            c.check(window, sinks)
        else:
            assert torch.equal(c.out, want), (window, sinks)


@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
@pytest.mark.parametrize("idle", [0, 30])
@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 4, 3), (20, 3), (0, 0)])
def test_tokens_before_position_zero_under_any_window(torch, window, sinks, idle, fmt, dtype):
    """Lengths shorter than the new tokens: the tokens at positions below 0 see nothing, the others
    what they see in any case, however near the window is to the largest number."""
    lens, new = [2, 70, 1, 40] + [0] * idle, [9, 5, 12, 70 - idle] + [0] * idle
    c = Case(torch, lens, new, 4, 2, 64, 16, fmt, dtype, seed=17)
    c.check(window, sinks)
    rows = c.out[:9]
    assert (rows[:7] == 0).all() and (rows[7:] != 0).any(dim=1).all()


@pytest.mark.parametrize("new", [1, 33])
def test_in_place_over_the_queries(torch, new):
    c = Case(torch, [900, 300], [new, new], 4, 2, 64, 16, "bf16", "bf16", seed=8)
    c.device()
    c.call()
    want = c.out.clone()
    c.call(out=c.dq)
    torch.cuda.synchronize()
    assert torch.equal(c.dq, want)


@pytest.mark.parametrize("lens,new", [([5000, 70, 1, 900], [1, 1, 1, 1]), ([3000, 200], [300, 1])])
def test_repeated_calls_give_the_same_bits(torch, lens, new):
    c = Case(torch, lens, new, 8, 2, 128, 32, "bf16", "bf16", seed=9)
    c.device()
    c.call()
    first = c.out.clone()
    for _ in range(3):
        c.ws.fill_(0x55)
        c.call()
        assert torch.equal(c.out, first)


def test_an_answer_does_not_depend_on_the_rest_of_the_batch(torch):
    """The same request alone and among others: split otherwise, the same within rounding."""
    c = Case(torch, [2000, 300, 5], [1, 1, 1], 8, 2, 128, 32, "bf16", "fp32", seed=10)
    c.check()
    whole = c.out.clone()
    c.R = c.T = 1
    c.call()
    assert (c.out[0] - whole[0]).abs().max() <= 1e-5 * whole[0].abs().max()


def test_offsets_past_32_bits(torch):
    """Pools of over 4 GB each, pages at their very end."""
    G, page, hd, n_pages = 8, 256, 128, 9000                    # 4.7 GB of keys, and of values
    pool = [torch.empty(n_pages, G, page, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    use = [8999, 0, 8500]
    rng = np.random.default_rng(11)
    small = round_bf16(rng.standard_normal((2, 3, G, page, hd)))
    slots = np.concatenate([p * page + np.arange(page) for p in use])
    cache = native.paged_cache("bf16", G, hd, page, n_pages, *pool)
    rows = [torch.from_numpy(small[i].transpose(0, 2, 1, 3).reshape(3 * page, G * hd).copy()).cuda().to(torch.bfloat16)
            for i in range(2)]
    native.apex_paged_store(cache, rows[0], rows[1], "bf16", 3 * page, G * hd, G * hd, i32(torch, slots))
    assert torch.equal(pool[0][8999].double().cpu(), torch.from_numpy(small[0, 0]))
    for new in (1, 40):
        q = round_bf16(rng.standard_normal((new, G, hd)))
        dq = torch.from_numpy(q.reshape(new, -1)).cuda().to(torch.bfloat16)
        out = torch.zeros_like(dq)
        n = native.apex_attention_paged_workspace_bytes(new, 1, G, G, hd)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        native.apex_attention_paged(cache, dq, "bf16", new, 1, G, G * hd, i32(torch, [0, new]), i32(torch, [700]),
                                    i32(torch, [use]), 3, 0, 0, hd ** -0.5, out, G * hd, ws, n)
        want, size, peak = opaged.attend(q, small[0], small[1], [0, new], [700], np.array([[0, 1, 2]]), 0, 0,
                                         hd ** -0.5, np.zeros_like(q))
        compare(out.double().cpu().numpy().reshape(q.shape), want, size, peak, hd, "bf16")


# ------------------------------------------------------------------------------------- store
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("T,G,hd,page", [(1, 1, 64, 16), (37, 3, 128, 16), (130, 8, 64, 64), (5, 2, 128, 1024)])
def test_store(torch, T, G, hd, page, fmt, dtype):
    rng = np.random.default_rng(T)
    n_pages = cdiv(T, page) + 2
    slots = rng.permutation(n_pages * page)[:T].astype(np.int64)
    if T > 3:
        slots[1], slots[3] = -1, n_pages * page                      # left out
    x = rng.standard_normal((2, T, G, hd)) * np.exp(rng.uniform(-20, 20, (2, T, G, 1)))
    x[0, T // 2, 0] = 0.0                                            # a row of zeros
    x[1, 0, 0, :8] = x[1, 0, 0, 8]                                   # equal values
    # ties between codes: the largest value 448 * 2^-5 makes the scale 2^-5
    tie = np.array([0.5, 1.5, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 248.0, 464.0 - 24]) * 2.0 ** -5
    x[0, T - 1, G - 1], x[0, T - 1, G - 1, :8], x[0, T - 1, G - 1, 9] = 0, tie, -448 * 2.0 ** -5
    x = round_bf16(x) if dtype == "bf16" else x.astype(np.float32).astype(np.float64)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    pools, scales, refs, ref_scales = [], [None] * 2, [], [None] * 2
    for i in range(2):
        if fmt == "bf16":
            pools.append(torch.full((n_pages, G, page, hd), 5.0, dtype=torch.bfloat16, device="cuda"))
            refs.append(np.full((n_pages, G, page, hd), 5.0))
        else:
            pools.append(torch.full((n_pages, G, page, hd), 0x31, dtype=torch.uint8, device="cuda"))
            refs.append(np.full((n_pages, G, page, hd), 0x31, np.uint8))
            scales[i] = torch.full((n_pages, G, page), 9.0, device="cuda")
            ref_scales[i] = np.full((n_pages, G, page), 9.0, np.float32)
        opaged.store(x[i], slots, page, refs[i], ref_scales[i])
    cache = native.paged_cache(fmt, G, hd, page, n_pages, *pools, *scales)
    wide = torch.from_numpy(np.concatenate([x[0].reshape(T, -1), x[1].reshape(T, -1)], 1)).cuda().to(t)
    k, v = wide[:, :G * hd], wide[:, G * hd:]
    native.apex_paged_store(cache, k, v, dtype, T, k.stride(0), v.stride(0), i32(torch, slots))
    torch.cuda.synchronize()
    for i in range(2):
        if fmt == "bf16":
            assert np.array_equal(pools[i].double().cpu().numpy(), refs[i])
        else:
            assert np.array_equal(scales[i].cpu().numpy(), ref_scales[i])
            # a code of -0 for a value of -0 is as good
            got, want = pools[i].cpu().numpy(), refs[i]
            same = (got == want) | ((got & 0x7F == 0) & (want & 0x7F == 0))
            assert same.all(), (np.argwhere(~same)[:5], got[~same][:5], want[~same][:5])


def test_store_of_rows_that_are_not_finite(torch):
    x = torch.ones(3, 64, device="cuda")
    x[0, 5], x[1, 63] = float("inf"), float("nan")
    codes = [torch.zeros(1, 1, 16, 64, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(1, 1, 16, device="cuda") for _ in range(2)]
    cache = native.paged_cache("fp8", 1, 64, 16, 1, *codes, *scales)
    native.apex_paged_store(cache, x, x, "fp32", 3, 64, 64, i32(torch, [0, 1, 2]))
    assert torch.isnan(scales[0][0, 0, :2]).all() and scales[1][0, 0, 2] == torch.tensor(1 / 448, dtype=torch.float32)
    assert (codes[0][0, 0, 2] == 0x7E).all() and (codes[0][0, 0, :2] == 0).all()


def test_store_of_tiny_rows(torch):
    x = np.zeros((4, 64), np.float32)
    x[0, :4] = [2e-38, 1e-38, -7e-39, 1e-39]
    x[1, :4] = [1e-40, -5e-41, 3e-42, 0]
    x[2, 0] = 1e-44                                                  # the scale rounds to 0
    x[3, :2] = [3.3e38, 1.0]
    codes = [torch.zeros(1, 1, 16, 64, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(1, 1, 16, device="cuda") for _ in range(2)]
    cache = native.paged_cache("fp8", 1, 64, 16, 1, *codes, *scales)
    d = torch.from_numpy(x).cuda()
    native.apex_paged_store(cache, d, d, "fp32", 4, 64, 64, i32(torch, [0, 1, 2, 3]))
    ref, ref_s = np.zeros((1, 1, 16, 64), np.uint8), np.zeros((1, 1, 16), np.float32)
    opaged.store(x.astype(np.float64)[:, None], [0, 1, 2, 3], 16, ref, ref_s)
    assert np.array_equal(scales[0].cpu().numpy(), ref_s)
    assert np.array_equal(codes[0].cpu().numpy(), ref)


# -------------------------------------------------------------------------------------- plan
class PlanCall:
    def __init__(self, torch, R, n_pages, nb, T):
        z = lambda *s: torch.full(s, 77, dtype=torch.int32, device="cuda")
        self.seq, self.cu, self.slots, self.pos, self.count_out, self.status = (
            z(R), z(R + 1), z(T), z(T), z(1), z(R))

    def run(self, torch, cached, n_new, page, n_pages, table, T, free, count, stream=None):
        self.table, self.free = i32(torch, table), i32(torch, free)
        self.args = (i32(torch, cached), i32(torch, n_new), len(cached), page, n_pages, table.shape[1], T, self.free,
                     i32(torch, [count]), self.table, self.seq, self.cu, self.slots, self.pos, self.count_out,
                     self.status, stream)
        native.apex_paged_plan(*self.args)

    def check(self, want):
        for got, name in ((self.table, "block_table"), (self.free, "free_pages"), (self.seq, "seq_len"),
                          (self.cu, "cu_new"), (self.slots, "slot_map"), (self.pos, "positions"),
                          (self.status, "status")):
            assert np.array_equal(got.cpu().numpy(), want[name]), name
        assert int(self.count_out[0]) == want["free_count"]


@pytest.mark.parametrize("R,page,nb,n_pages,T,longest", [
    (1, 16, 1, 1, 1, 1), (5, 16, 9, 30, 40, 30), (64, 32, 20, 700, 300, 5), (64, 16, 20, 300, 200, 60),
    (1000, 64, 7, 3000, 2500, 4), (1025, 16, 9, 4000, 9000, 40), (4096, 16, 5, 9000, 5000, 3)])
def test_plan_over_steps(torch, R, page, nb, n_pages, T, longest):
    """Steps of a server: each takes the tables, lengths and free pages that the one before left."""
    rng = np.random.default_rng(R)
    table, cached = np.full((R, nb), -1), np.zeros(R, np.int64)
    free, count = rng.permutation(n_pages), n_pages
    call = PlanCall(torch, R, n_pages, nb, T)
    for step in range(6):
        n_new = rng.integers(0, longest + 1, R)
        n_new[rng.random(R) < 0.1] = -1
        if step == 3:
            n_new[rng.integers(0, R)] = nb * page + 1                # more than a row has
        call.run(torch, cached, n_new, page, n_pages, table, T, free, count)
        want = opaged.plan(cached, n_new, page, n_pages, table, T, free, count)
        call.check(want)
        native.apex_paged_plan(*call.args)                           # the same inputs again
        call.check(want)
        table, cached, free, count = want["block_table"], want["seq_len"], want["free_pages"], want["free_count"]


def test_plan_of_numbers_that_make_no_sense(torch):
    big = 2 ** 31 - 1
    table = np.array([[3, 99], [-5, 1], [0, 1], [2, -1], [-1, -1], [-1, -1]])
    cached = [20, 30, -7, big, 0, 0]
    n_new = [2, 1, 3, big, -9, big]
    for count in (-4, 3, 10 ** 6):
        call = PlanCall(torch, 6, 4, 2, 8)
        free = [-8, 2, 77, 1]
        call.run(torch, cached, n_new, 16, 4, table, 8, free, count)
        call.check(opaged.plan(cached, n_new, 16, 4, table, 8, free, count))


def test_plan_of_inputs_in_one_buffer(torch):
    """Lengths that are the new tokens as well (each request doubles), and the count of free pages
    among them."""
    n = [9, 16, 0, 17, 3]
    table = np.array([[0, -1, -1], [1, -1, -1], [-1, -1, -1], [2, 3, -1], [4, -1, -1]])
    free = [5, 6, 7, 8, 9, 10, 11, 12]
    call = PlanCall(torch, 5, 13, 3, 60)
    call.table, call.free = i32(torch, table), i32(torch, free + [0] * 5)
    one = i32(torch, n + [8])
    native.apex_paged_plan(one, one, 5, 16, 13, 3, 60, call.free, one[5:], call.table, call.seq, call.cu, call.slots,
                           call.pos, call.count_out, call.status)
    call.check(opaged.plan(n, n, 16, 13, table, 60, free + [0] * 5, 8))
    call = PlanCall(torch, 1, 13, 3, 60)                             # all three the same word
    call.table, call.free, one = i32(torch, [[0, -1, -1]]), i32(torch, list(range(1, 14))), i32(torch, [7])
    native.apex_paged_plan(one, one, 1, 16, 13, 3, 60, call.free, one, call.table, call.seq, call.cu, call.slots,
                           call.pos, call.count_out, call.status)
    call.check(opaged.plan([7], [7], 16, 13, np.array([[0, -1, -1]]), 60, list(range(1, 14)), 7))


def test_plan_without_requests_or_rows(torch):
    call = PlanCall(torch, 0, 4, 2, 5)
    free, count = i32(torch, [0, 1, 2, 3]), i32(torch, [3])
    native.apex_paged_plan(None, None, 0, 16, 4, 2, 5, free, count, None, None, call.cu, call.slots, call.pos,
                           call.count_out, None)
    assert int(call.cu[0]) == 0 and (call.slots == -1).all() and int(call.count_out[0]) == 3
    table = np.array([[1, -1]])
    call = PlanCall(torch, 1, 4, 2, 0)
    call.run(torch, [5], [2], 16, 4, table, 0, [0, 2, 3, 0], 3)      # no row is left for it
    call.check(opaged.plan([5], [2], 16, 4, table, 0, [0, 2, 3, 0], 3))


# -------------------------------------------------------------------------------- all of them
@pytest.mark.parametrize("fmt,dtype", FORMATS, ids=FMT_IDS)
def test_a_server_from_prompts_to_tokens(torch, fmt, dtype):
    """Plan, store and attention as a server calls them: prompts in chunks, then single tokens,
    requests that end and begin; every step's attention against the oracle over all keys and
    values so far.  Run on a stream of its own, the steps captured once and replayed."""
    R, page, nb, G, H, hd, n_pages, T = 4, 16, 8, 2, 6, 64, 24, 40
    rng = np.random.default_rng(20)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    pages = [torch.zeros(n_pages, G, page, hd, dtype=torch.bfloat16 if fmt == "bf16" else torch.uint8, device="cuda")
             for _ in range(2)]
    scales = [torch.zeros(n_pages, G, page, device="cuda") if fmt == "fp8" else None for _ in range(2)]
    cache = native.paged_cache(fmt, G, hd, page, n_pages, *pages, *scales)
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    cached, n_new, seq, cu, slots, count, count_out = z(R), z(R), z(R), z(R + 1), z(T), z(1), z(1)
    table, free, status, positions = z(R, nb) - 1, torch.arange(n_pages, dtype=torch.int32, device="cuda"), z(R), z(T)
    count.fill_(n_pages)
    qkv = torch.zeros(T, (H + 2 * G) * hd, dtype=t, device="cuda")
    out = torch.zeros(T, H * hd, dtype=t, device="cuda")
    n = native.apex_attention_paged_workspace_bytes(T, R, H, G, hd)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()

    def step():
        s = torch.cuda.current_stream().cuda_stream
        native.apex_paged_plan(cached, n_new, R, page, n_pages, nb, T, free, count, table, seq, cu, slots, positions,
                               count_out, status, s)
        k, v = qkv[:, H * hd:(H + G) * hd], qkv[:, (H + G) * hd:]
        native.apex_paged_store(cache, k, v, dtype, T, k.stride(0), v.stride(0), slots, s)
        native.apex_attention_paged(cache, qkv, dtype, T, R, H, qkv.stride(0), cu, seq, table, nb, 40, 3, 0.125, out,
                                    out.stride(0), ws, n, s)
        cached.copy_(seq)
        count.copy_(count_out)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    cached.zero_()
    count.fill_(n_pages)
    host = dict(cached=np.zeros(R, np.int64), table=np.full((R, nb), -1), free=np.arange(n_pages), count=n_pages)
    ref = [np.zeros((n_pages, G, page, hd), np.float64 if fmt == "bf16" else np.uint8) for _ in range(2)]
    ref_s = [np.zeros((n_pages, G, page), np.float32) if fmt == "fp8" else None for _ in range(2)]
    chunks = [[20, 1, 0, 9], [20, 1, 5, 9], [1, 1, 1, 1], [1, 1, 1, -1], [1, -1, 1, 33], [1, 7, 1, 1], [1, 1, 1, 1],
              [-1, 30, 1, 2], [12, 1, 1, 1]]
    for i, new in enumerate(chunks):
        x = rng.standard_normal((T, H + 2 * G, hd))
        x = round_bf16(x) if dtype == "bf16" else x.astype(np.float32).astype(np.float64)
        qkv.copy_(torch.from_numpy(x.reshape(T, -1)))
        n_new.copy_(i32(torch, new))
        out.fill_(7.0)
        torch.cuda.synchronize()
        if i % 3 == 2:
            step()                                   # eager calls among the replays
        else:
            graph.replay()
        torch.cuda.synchronize()
        want = opaged.plan(host["cached"], new, page, n_pages, host["table"], T, host["free"], host["count"])
        assert np.array_equal(table.cpu().numpy(), want["block_table"])
        assert np.array_equal(slots.cpu().numpy(), want["slot_map"]) and int(count[0]) == want["free_count"]
        host = dict(cached=want["seq_len"], table=want["block_table"], free=want["free_pages"], count=want["free_count"])
        for kv, lo in ((0, H), (1, H + G)):
            opaged.store(x[:, lo:lo + G], want["slot_map"], page, ref[kv], ref_s[kv])
        K, V = ref if fmt == "bf16" else [fp8.decode_array(c) * s[..., None].astype(np.float64) for c, s in zip(ref, ref_s)]
        ref_out, size, peak = opaged.attend(x[:, :H], K, V, want["cu_new"], want["seq_len"], want["block_table"], 40, 3,
                                            0.125, np.full((T, H, hd), 7.0))
        got = out.double().cpu().numpy().reshape(T, H, hd)
        compare(got, ref_out, size, peak, hd, dtype)


def test_readme_example_runs(torch):
    """The Python example of README.md for the paged cache, run as written."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "README.md")).read()
    code = re.search(r"<!-- example: paged -->\s*```python\n(.*?)```", text, re.S).group(1)
    exec(compile(code, "README.md example", "exec"), {})


def test_two_streams_with_workspaces_of_their_own(torch):
    a = Case(torch, [3000, 50], [1, 1], 8, 2, 128, 16, "bf16", "bf16", seed=30)
    b = Case(torch, [900, 400], [100, 7], 8, 2, 128, 16, "fp8", "bf16", seed=31)
    a.device(), b.device()
    a.call(), b.call()
    torch.cuda.synchronize()
    want = a.out.clone(), b.out.clone()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        a.call(stream=streams[0].cuda_stream)
        b.call(stream=streams[1].cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])


def test_two_graphs_that_share_a_workspace(torch):
    """Replayed in turn on one stream, with eager calls between: nothing in the workspace is kept
    from one call for the next."""
    a = Case(torch, [4000, 50], [1, 1], 8, 2, 128, 16, "bf16", "bf16", seed=32)
    b = Case(torch, [2900, 400], [100, 7], 8, 2, 128, 16, "fp8", "bf16", seed=33)
    a.device(), b.device()
    a.ws = b.ws = max(a.ws, b.ws, key=lambda w: w.numel())
    a.call(), b.call()
    torch.cuda.synchronize()
    want = a.out.clone(), b.out.clone()
    graphs = []
    for c in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.call(stream=torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    for i in range(4):
        a.out.zero_(), b.out.zero_()
        if i == 2:
            a.ws.fill_(0x55)
        for g in graphs if i % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])
        b.call(out=b.out)
        torch.cuda.synchronize()
        assert torch.equal(b.out, want[1])
