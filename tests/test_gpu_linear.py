"""Projection by 4-bit weights against the float64 oracle.

Tolerances.  Per output, with size = sum |s| (32 + q + |z|) |x| (plus |bias| and |residual|): every product is exact
(5 bits times 8), and a group's two sums of products and the sum over groups are at most P * group + K / 32 + 40 additions
(P = 3 pieces of fp32 values, else 1), each off by at most 2^-24 of a partial sum that `size` bounds.  A bf16 result adds
half a step, 2^-8 of it, an fp32 one 2^-24.  That bound is for each output.  Over all outputs the 2-norm of the error is
much smaller, as roundings are independent and partial sums of the values of mixed signs here grow with the root of their
number: sums of n terms of rms 24 |x| round with an rms of 2^-24 * 0.4 * 24 |x| sqrt(n) each, sqrt(n / 2) of them like the
last, which is 1e-6 of the result's sqrt(n) * 4.6 |x| for n = 128, 1.5e-6 with the sum of x as well and at most 2.6e-6 with
the additions of three pieces: fp32 at most 3e-6, where a lost third piece would leave 7e-6.  bf16 rounds once, with an
rms of at most 2^-8 / sqrt(3) * 0.72 = 1.63e-3: 2e-3.
"""
import os
import re

import numpy as np
import pytest

from oracle import linear_w4
from paper_2608_11688_amd import native

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available()
    native.lib()
    return t


class Case:
    def __init__(self, torch, T, N, K, group, x="bf16", y="bf16", bias=False, residual=False, seed=0, extra=0):
        self.torch, self.T, self.N, self.K, self.group, self.x_type, self.y_type = torch, T, N, K, group, x, y
        rng = np.random.default_rng(seed)
        groups = linear_w4.padded(K) // group
        self.q = rng.integers(0, 16, (N, K))
        self.s = linear_w4.bf16(((rng.random((N, groups)) + 0.5) * 0.05).astype(np.float32))
        self.z = linear_w4.bf16(rng.integers(5, 11, (N, groups)).astype(np.float32))
        self.x = self.rounded(rng.standard_normal((T, K)), x)
        self.b = rng.standard_normal(N).astype(np.float32) if bias else None
        self.r = self.rounded(rng.standard_normal((T, N)), y) if residual else None
        self.extra = extra

    @staticmethod
    def rounded(v, kind):
        v = v.astype(np.float32)
        return linear_w4.bf16(v) if kind == "bf16" else v.astype(np.float64)

    def type(self, kind):
        return self.torch.bfloat16 if kind == "bf16" else self.torch.float32

    def rows(self, v, kind, fill):
        """On the GPU, with `extra` values of `fill` behind every row."""
        wide = self.torch.full((v.shape[0], v.shape[1] + self.extra), fill, dtype=self.type(kind), device="cuda")
        wide[:, :v.shape[1]] = self.torch.from_numpy(np.ascontiguousarray(v)).cuda().to(self.type(kind))
        return wide

    def device(self):
        torch = self.torch
        self.dw = torch.from_numpy(linear_w4.pack(self.q, self.s, self.z)).cuda()
        assert self.dw.numel() == native.apex_linear_w4_bytes(self.N, self.K, self.group)
        self.dx = self.rows(self.x, self.x_type, float("nan"))     # what stands between rows is not read
        self.db = None if self.b is None else torch.from_numpy(self.b).cuda()
        self.dr = None if self.r is None else self.rows(self.r, self.y_type, 5.0)
        self.dy = torch.full((self.T, self.N + self.extra), 7.0, dtype=self.type(self.y_type), device="cuda")
        n = native.apex_linear_w4_workspace_bytes(self.T, self.N, self.K, self.group, self.x_type)
        self.ws = torch.full((n + 64,), 0xAB, dtype=torch.uint8, device="cuda")
        return self

    def call(self, stream=None, y=None):
        y = self.dy if y is None else y
        native.apex_linear_w4(self.dw, self.N, self.K, self.group, self.dx, self.x_type, self.T, self.dx.stride(0),
                              self.db, self.dr, self.dr.stride(0) if self.dr is not None else 0, y, self.y_type,
                              y.stride(0), self.ws, self.ws.numel() - 64, stream)

    def check(self, norm=True):
        self.device()
        self.call()
        self.torch.cuda.synchronize()
        assert (self.dy[:, self.N:] == 7).all() and (self.ws[-64:] == 0xAB).all()
        return self.compare(self.dy, norm)

    def compare(self, y, norm=True):
        got = y[:, :self.N].double().cpu().numpy()
        with np.errstate(invalid="ignore", over="ignore"):
            want, size = linear_w4.apply(self.x, self.q, self.s, self.z, self.group, self.b, self.r)
        return compare(got, want, size, self.group, self.K, self.x_type, self.y_type, norm)


def compare(got, want, size, group, K, x_type, y_type, norm=True):
    bad = ~np.isfinite(want)
    assert np.array_equal(np.isnan(got), bad)
    step = 2.0 ** -8 if y_type == "bf16" else 2.0 ** -24
    adds = (3 if x_type == "fp32" else 1) * group + K / 32 + 40
    err = np.abs(got - want)
    bound = size * adds * 2.0 ** -24 + np.abs(want) * step
    assert (err[~bad] <= bound[~bad]).all(), (err[~bad] - bound[~bad]).max()
    rel = np.linalg.norm(err[~bad]) / max(np.linalg.norm(want[~bad]), 1e-30)
    if norm:
        assert rel <= (2e-3 if y_type == "bf16" else 3e-6), rel
    return rel


TYPES = [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "bf16"), ("fp32", "fp32")]
TYPE_IDS = ["-".join(t) for t in TYPES]

# T, N, K, group, bias, residual, extra values in a row
CASES = [
    (1, 16, 128, 128, False, False, 0), (1, 1, 8, 32, True, True, 0), (1, 17, 40, 32, False, True, 8),
    (1, 100, 1000, 64, True, False, 16), (1, 2048, 1024, 64, False, False, 0), (1, 33, 4104, 128, True, True, 0),
    (2, 37, 96, 32, False, False, 0), (3, 50, 264, 128, True, True, 8), (4, 130, 520, 64, False, True, 0),
    (5, 64, 2048, 32, False, False, 0), (7, 1031, 1416, 32, True, False, 0), (8, 48, 256, 64, False, False, 8),
    (9, 31, 136, 128, False, True, 0), (15, 65, 384, 64, True, True, 0), (16, 16, 640, 32, False, False, 0),
    (17, 95, 512, 128, False, True, 8), (31, 129, 360, 64, True, False, 0), (32, 512, 1024, 64, False, True, 0),
    (33, 63, 128, 32, True, True, 8), (48, 100, 776, 128, False, False, 0), (63, 257, 256, 32, False, False, 0),
    (64, 64, 1152, 64, True, True, 0), (65, 127, 400, 128, False, False, 8), (100, 300, 512, 64, True, True, 0),
    (127, 129, 264, 32, False, True, 0), (128, 128, 256, 128, False, False, 0), (129, 255, 640, 64, True, False, 8),
    (200, 77, 1000, 32, False, False, 0), (256, 256, 384, 128, False, True, 0), (300, 511, 136, 64, True, True, 0),
    (513, 260, 904, 128, True, True, 8),
]


@pytest.mark.parametrize("x,y", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("T,N,K,group,bias,residual,extra", CASES, ids=[str(c) for c in CASES])
def test_projection(torch, T, N, K, group, bias, residual, extra, x, y):
    print(Case(torch, T, N, K, group, x, y, bias, residual, seed=T + N, extra=extra).check(norm=T * N >= 1000))


class Large:
    """Sizes of the product in tiles, its reference in float64 on the GPU."""

    def __init__(self, torch, T, N, K, group, x, y, bias=False, residual=False, extra=0, seed=0):
        self.torch, self.T, self.N, self.K, self.group, self.x_type, self.y_type = torch, T, N, K, group, x, y
        gen = torch.Generator(device="cuda").manual_seed(seed)
        types = {"bf16": torch.bfloat16, "fp32": torch.float32}
        n = native.apex_linear_w4_bytes(N, K, group)
        Kp = linear_w4.padded(K)
        self.w = torch.randint(0, 256, (n,), dtype=torch.uint8, generator=gen, device="cuda")
        words = self.w[N * Kp // 2:].view(torch.bfloat16).view(Kp // group, N, 2)
        words[..., 0] = torch.randint(5, 11, words.shape[:2], generator=gen, device="cuda").bfloat16()
        words[..., 1] = (torch.rand(words.shape[:2], generator=gen, device="cuda") * 0.05 + 0.02).bfloat16()
        self.x = torch.full((T, K + extra), float("nan"), dtype=types[x], device="cuda")
        self.x[:, :K] = torch.randn(T, K, generator=gen, device="cuda")
        self.b = torch.randn(N, generator=gen, device="cuda") if bias else None
        self.r = torch.randn(T, N + extra, generator=gen, device="cuda").to(types[y]) if residual else None
        self.y = torch.full((T, N + extra), 7.0, dtype=types[y], device="cuda")
        need = native.apex_linear_w4_workspace_bytes(T, N, K, group, x)
        self.ws = torch.full((need + 64,), 0xAB, dtype=torch.uint8, device="cuda")

    def call(self, stream=None):
        native.apex_linear_w4(self.w, self.N, self.K, self.group, self.x, self.x_type, self.T, self.x.stride(0), self.b, self.r,
                              self.r.stride(0) if self.r is not None else 0, self.y, self.y_type, self.y.stride(0), self.ws,
                              self.ws.numel() - 64, stream)

    def reference(self):
        torch, N, K, Kp = self.torch, self.N, self.K, linear_w4.padded(self.K)
        code = self.w[:N * Kp // 2].view(torch.int32).view(N, Kp // 128, 4, 4)      # [row, block, a, j]
        q = torch.stack([code >> (4 * (e // 2) + 16 * (e % 2)) & 15 for e in range(8)], -1)
        q = q.transpose(2, 3).reshape(N, Kp)[:, :K].double()
        words = self.w[N * Kp // 2:].view(torch.bfloat16).view(Kp // self.group, N, 2).double()
        z, s = (words[..., i].t().repeat_interleave(self.group, 1)[:, :K] for i in (0, 1))
        x = self.x[:, :K].double()
        want = x @ (s * (q - z)).t().contiguous()
        size = x.abs() @ (s.abs() * (32 + q + z.abs())).t().contiguous()
        for extra in (self.b, self.r[:, :N] if self.r is not None else None):
            if extra is not None:
                want, size = want + extra.double(), size + extra.double().abs()
        return want.cpu().numpy(), size.cpu().numpy()

    def check(self):
        self.call()
        self.torch.cuda.synchronize()
        self.in_tiles = bool((self.ws[:256] != 0xAB).any())     # x in the order of the tiles
        assert (self.y[:, self.N:] == 7).all() and (self.ws[-64:] == 0xAB).all()
        return self.compare()

    def check_rows(self, T):
        """The first T rows of y, and that the others stay."""
        self.call()
        self.torch.cuda.synchronize()
        assert (self.y[T:] == 7).all() and (self.ws[-64:] == 0xAB).all()
        y, self.y = self.y, self.y[:T]
        self.compare()
        self.y = y

    def compare(self):
        want, size = self.reference()
        return compare(self.y[:, :self.N].double().cpu().numpy(), want, size, self.group, self.K, self.x_type, self.y_type)


# T, N, K, group, types of x and y, bias, residual, extra values in a row
LARGE = [
    (33, 7000, 8136, 128, "bf16", "bf16", False, False, 0), (64, 14337, 4096, 32, "bf16", "fp32", True, True, 8),
    (63, 9000, 6912, 64, "bf16", "bf16", True, False, 16), (65, 14999, 7688, 32, "bf16", "bf16", False, True, 0),
    (33, 25000, 5400, 64, "fp32", "fp32", False, True, 0), (48, 3333, 6016, 128, "fp32", "bf16", True, False, 8),
    (100, 6052, 3840, 32, "fp32", "fp32", True, True, 0), (129, 9001, 7936, 128, "bf16", "fp32", False, False, 0),
    (300, 2816, 4104, 64, "bf16", "bf16", True, True, 8), (513, 5121, 1416, 128, "bf16", "bf16", False, True, 0),
    (2050, 4100, 520, 32, "bf16", "fp32", False, False, 0),       # more tiles than a round, shares behind it
    (2048, 4096, 512, 128, "bf16", "bf16", False, False, 0),      # a round of whole tiles and nothing behind it
    (1700, 4001, 392, 64, "fp32", "bf16", True, True, 0),
    (1300, 255, 20000, 64, "bf16", "fp32", False, False, 0), (4000, 600, 24000, 128, "bf16", "bf16", False, True, 0),
    (70000, 250, 232, 64, "bf16", "bf16", False, False, 0),       # many tiles of few steps
    (2300, 4100, 1160, 32, "fp32", "bf16", True, True, 8), (1150, 5051, 776, 64, "bf16", "bf16", True, True, 8),
    (2200, 6100, 2600, 64, "bf16", "fp32", False, True, 0), (8190, 600, 2056, 32, "bf16", "bf16", True, False, 0),
    (2048, 4096, 9000, 32, "bf16", "fp32", False, False, 0), (64, 60000, 9000, 32, "bf16", "bf16", False, True, 0),   # many groups
]
# tiles of wavefronts: more rows than one tile, with 1 to 8 wavefronts along K
SOME = [
    (65, 4999, 7688, 32, "bf16", "bf16", False, True, 0), (17, 5000, 5400, 64, "fp32", "fp32", False, True, 0),
    (100, 2052, 3840, 32, "fp32", "fp32", True, True, 0), (129, 3001, 7936, 128, "bf16", "fp32", False, False, 0),
    (800, 255, 20000, 64, "bf16", "fp32", False, False, 0), (3000, 60, 24000, 128, "bf16", "bf16", False, True, 0),
    (1073, 1288, 128, 32, "bf16", "fp32", True, True, 8), (2001, 510, 256, 64, "bf16", "bf16", False, True, 0),
    (353, 4099, 232, 128, "bf16", "bf16", False, False, 8), (901, 803, 160, 32, "fp32", "fp32", True, True, 0),
    (399, 600, 1000, 64, "fp32", "bf16", False, False, 0), (100, 5000, 128, 128, "fp32", "fp32", False, True, 0),
    (9999, 40, 520, 32, "bf16", "fp32", True, False, 0), (86, 22171, 256, 128, "bf16", "bf16", False, True, 0),
    (1 << 20, 5, 40, 32, "fp32", "fp32", False, False, 0),        # the most rows
]


@pytest.mark.parametrize("case", LARGE, ids=[str(c) for c in LARGE])
def test_products_in_tiles(torch, case):
    c = Large(torch, *case, seed=case[0])
    print(c.check())
    assert c.in_tiles


@pytest.mark.parametrize("case", SOME, ids=[str(c) for c in SOME])
def test_tiles_of_wavefronts(torch, case):
    c = Large(torch, *case, seed=case[0])
    print(c.check())
    assert not c.in_tiles


def test_two_graphs_that_share_a_workspace(torch):
    """Replayed in turn on one stream, with eager calls between: nothing in the workspace is kept from call to call."""
    a = Large(torch, 300, 2816, 4104, 64, "bf16", "fp32", seed=1)
    b = Large(torch, 129, 9001, 2000, 128, "fp32", "bf16", seed=2)
    a.ws = b.ws = torch.empty(max(a.ws.numel(), b.ws.numel()), dtype=torch.uint8, device="cuda")
    want = []
    for c in (a, b):
        c.call()
        torch.cuda.synchronize()
        want.append(c.y.clone())
    side, graphs = torch.cuda.Stream(), [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.stream(side):
        for c, graph in zip((a, b), graphs):
            with torch.cuda.graph(graph, stream=side):
                c.call(side.cuda_stream)
    for i in range(4):
        for c, graph, right in zip((a, b), graphs, want):
            c.y.fill_(7.0)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(c.y, right)
        b.call()
        torch.cuda.synchronize()
        assert torch.equal(b.y, want[1])


def test_a_workspace_serves_fewer_rows(torch):
    """One workspace of the largest T, and what stands behind it, through every T below."""
    N, K, T = 1500, 2048, 700
    c = Large(torch, T, N, K, 32, "bf16", "fp32")
    x = c.x
    for c.T in (700, 513, 300, 129, 64, 33, 1):
        c.x = x[:c.T]
        c.y.fill_(7.0)
        c.check_rows(c.T)


@pytest.mark.parametrize("case", [LARGE[1], LARGE[6], LARGE[8], LARGE[10]], ids=str)
def test_products_in_tiles_captured_and_replayed(torch, case):
    c = Large(torch, *case, seed=1)
    c.call()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            c.call(side.cuda_stream)
    for i in range(3):
        c.x[:, :c.K] = torch.randn(c.T, c.K, device="cuda")
        c.ws[:-64].fill_(i)
        c.y.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = c.y.clone()
        c.y.fill_(7.0)
        c.call()
        torch.cuda.synchronize()
        assert torch.equal(replayed, c.y)
    c.check()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_not_finite_in_tiles(torch, value):
    c = Large(torch, 300, 2816, 4104, 64, "bf16", "fp32")
    c.call()
    clean = c.y.clone()
    c.x[137, 4000], c.x[299, 0] = value, value
    c.call()
    bad = torch.zeros(300, dtype=torch.bool, device="cuda")
    bad[[137, 299]] = True
    assert c.y[bad].isnan().all() and torch.equal(c.y[~bad], clean[~bad])


@pytest.mark.parametrize("T", [1, 5, 40, 150])
@pytest.mark.parametrize("x", ["bf16", "fp32"])
def test_residual_in_place_and_repeated(torch, T, x):
    c = Case(torch, T, 200, 520, 32, x, "fp32", True, True, seed=T).device()
    keep = c.dr.clone()
    c.call()
    first = c.dy.clone()
    c.call(y=c.dr)
    assert torch.equal(c.dr, first)               # the residual's own rows as the output
    c.dr.copy_(keep)
    c.ws.fill_(0xFF)
    c.call()
    assert torch.equal(c.dy, first)
    c.compare(first)


@pytest.mark.parametrize("T", [1, 3, 20, 70, 300])
@pytest.mark.parametrize("x", ["bf16", "fp32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_not_finite(torch, T, x, value):
    c = Case(torch, T, 70, 264, 64, x, "fp32", seed=T)
    c.x[T // 2, 77] = value
    c.device()
    c.call()
    got = c.dy.double().cpu().numpy()
    assert np.isnan(got[T // 2]).all()
    c.x[T // 2] = 0
    c.device()
    c.call()
    rest = np.arange(T) != T // 2
    assert np.array_equal(got[rest], c.dy.double().cpu().numpy()[rest])
    c.compare(c.dy, norm=False)


@pytest.mark.parametrize("T", [1, 20, 130])
def test_scales_of_any_kind(torch, T):
    c = Case(torch, T, 80, 300 // 8 * 8, 32, "bf16", "fp32", seed=9)
    c.s[3], c.z[3] = 0.0, 0.0                     # a row of zeros
    c.s[4, 1] = 0.0
    c.s[5] *= -1.0
    c.s[6] = linear_w4.bf16(np.float32(1e-30))
    c.s[7] = linear_w4.bf16(np.float32(1e30))
    c.z[8] = linear_w4.bf16(np.float32(-3.625))   # zero points outside of the codes and between them
    c.z[9] = linear_w4.bf16(np.float32(200.0))
    c.s[10, 2] = np.nan
    c.check(norm=False)
    assert (c.dy[:, 3] == 0).all()


@pytest.mark.parametrize("x", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 2, 20, 200])
def test_values_of_any_size(torch, T, x):
    c = Case(torch, T, 60, 400, 128, x, "fp32", seed=11)
    c.x = c.rounded(c.x * 2.0 ** np.random.default_rng(1).integers(-90, 100, c.x.shape), x)
    c.check(norm=False)
    c.x[:] = 0
    c.check(norm=False)
    assert (c.dy == 0).all()


@pytest.mark.parametrize("x", ["bf16", "fp32"])
@pytest.mark.parametrize("T,N", [(1, 3), (2, 40), (70, 20)])
def test_longest_rows(torch, T, N, x):
    print(Case(torch, T, N, 1 << 20, 128, x, "fp32", seed=5).check(norm=False))


def test_weights_past_32_bit_offsets(torch):
    N, K, group = 8300, 1 << 20, 128
    gen = torch.Generator(device="cuda").manual_seed(3)
    n = native.apex_linear_w4_bytes(N, K, group)
    w = torch.empty(n, dtype=torch.uint8, device="cuda")
    codes = w[:N * K // 2]
    for part in codes.split(1 << 30):
        part.copy_(torch.randint(0, 256, part.shape, dtype=torch.uint8, generator=gen, device="cuda"))
    words = w[N * K // 2:].view(torch.bfloat16).view(K // group, N, 2)
    words[..., 0] = 8.0
    words[..., 1] = 0.01
    x = torch.randn(2, K, generator=gen, device="cuda").bfloat16()
    y = torch.zeros(2, N, device="cuda")
    native.apex_linear_w4(w, N, K, group, x, "bf16", 2, K, None, None, 0, y, "fp32", N, None, 0)
    rows = [0, 1, 4095, 8191, 8192, N - 1]
    pick = torch.cat([codes.view(N, -1)[rows].reshape(-1), words[:, rows].contiguous().view(torch.uint8).reshape(-1)])
    q, s, z = linear_w4.unpack(pick.cpu().numpy(), len(rows), K, group)
    want, size = linear_w4.apply(x.double().cpu().numpy(), q, s, z, group)
    compare(y[:, rows].double().cpu().numpy(), want, size, group, K, "bf16", "fp32", norm=False)


@pytest.mark.parametrize("x,y", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("T", [1, 6, 33, 140])
def test_captured_and_replayed(torch, T, x, y):
    c = Case(torch, T, 150, 392, 64, x, y, True, True, seed=T).device()
    c.call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            c.call(stream=side.cuda_stream)
    for i in range(4):
        c.x = c.rounded(np.random.default_rng(i).standard_normal(c.x.shape), x)
        c.dx.copy_(c.rows(c.x, x, float("nan")))
        c.dy.fill_(7.0)
        c.ws.fill_(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = c.dy.clone()
        c.compare(replayed, norm=False)
        c.call()
        torch.cuda.synchronize()
        assert torch.equal(replayed, c.dy)


def test_two_streams_at_once(torch):
    a, b = (Case(torch, T, 1000, 2048, 64, "fp32", "fp32", seed=T).device() for T in (1, 90))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        a.call(streams[0].cuda_stream)
        b.call(streams[1].cuda_stream)
    torch.cuda.synchronize()
    a.compare(a.dy)
    b.compare(b.dy)


def test_a_chunk_agrees_with_its_rows(torch):
    """Rows alone and in a chunk: other orders of the same sums."""
    c = Case(torch, 130, 100, 640, 64, "fp32", "fp32", seed=2).device()
    c.call()
    c.compare(c.dy)
    whole = c.dy.clone()
    for t in (0, 64, 129):
        one = Case(torch, 1, 100, 640, 64, "fp32", "fp32", seed=2)
        one.x = c.x[t:t + 1]
        one.device()
        one.call()
        one.compare(one.dy, norm=False)
        assert torch.allclose(one.dy[0], whole[t], rtol=1e-4, atol=1e-4)


def test_packed_by_the_library(torch):
    rng = np.random.default_rng(8)
    w = linear_w4.bf16((rng.standard_normal((90, 200)) * 0.05).astype(np.float32))
    c = Case(torch, 3, 90, 200, 64, "fp32", "fp32", seed=8)
    c.q, c.s, c.z = linear_w4.quantise(w, 64)
    c.device()
    out = np.zeros(native.apex_linear_w4_bytes(90, 200, 64), np.uint8)
    native.apex_pack_linear_w4((w.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16), 90, 200, 64, out)
    c.dw = torch.from_numpy(out).cuda()
    c.call()
    c.compare(c.dy, norm=False)


def test_readme_example_runs(torch):
    """The Python example of README.md for projections and rotary positions, run as written."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "README.md")).read()
    code = re.search(r"<!-- example: projection -->\s*```python\n(.*?)```", text, re.S).group(1)
    exec(compile(code, "README.md example", "exec"), {})


def shifted_tolerance(group, K, pieces):
    """2-norm of the error of an fp32 result relative to the result's, for rows of x of any mean m and deviation d.  Of a
    group the sums go up to g (16 + q) x, 24 g (m^2 + d^2)^(1/2) at most in the root mean square, before the
    zero points' half, as large, is taken off; on the way there one instruction a 32 values and piece rounds sums that
    are half of that on average, and twice more round it whole, each by 2^-25 at most, 0.58 of that in the
    mean: 2^-25 * 0.58 * 24 g (pieces g / 32 / 4 + 2)^(1/2) r for a group, r = (m^2 + d^2)^(1/2).  An instruction
    may round within its 32 values too, 8 times, which multiplies its share by 8.  Groups' errors are independent, so a row
    has K / g of them in the square; the result's own size is s (q - z), 4.6 s for uniform codes around z, times r
    sqrt(K): the quotient has neither r nor K.  The additions over groups round sums no larger than the result, K / g of
    them, which is 2^-25 * 0.58 (K / g / 2)^(1/2)."""
    inside = 0.58 * 2.0 ** -25 * 24 * group * (8 * pieces * group / 128 + 2) ** 0.5 / (4.6 * group ** 0.5)
    over = 0.58 * 2.0 ** -25 * (K / group / 2) ** 0.5
    return inside + over


# T, N, K, group, type of x, in tiles
SHIFTED = [(300, 2816, 4104, 32, "bf16", True), (300, 2816, 4104, 64, "bf16", True), (300, 2816, 4104, 128, "bf16", True),
           (2050, 4100, 520, 32, "bf16", True), (64, 14337, 16384, 32, "bf16", True), (100, 6052, 3840, 32, "fp32", True),
           (100, 6052, 3840, 128, "fp32", True), (1700, 4001, 392, 64, "fp32", True), (65, 4999, 7688, 32, "bf16", False),
           (129, 3001, 7936, 128, "bf16", False), (100, 2052, 3840, 32, "fp32", False), (4, 3000, 4096, 32, "bf16", False),
           (1, 3000, 16384, 128, "bf16", False), (2, 3000, 4096, 64, "fp32", False)]


@pytest.mark.parametrize("mean,deviation", [(0.0, 1.0), (0.25, 1.0), (1.0, 1.0), (1.0, 0.3), (-10.0, 1.0)])
@pytest.mark.parametrize("case", SHIFTED, ids=str)
def test_rows_of_any_mean(torch, case, mean, deviation):
    """The codes' and the zero points' halves of a result grow with the mean of x, the result does not."""
    T, N, K, group, x, in_tiles = case
    c = Large(torch, T, N, K, group, x, "fp32", seed=T)
    Kp = linear_w4.padded(K)
    c.w[N * Kp // 2:].view(torch.bfloat16).view(Kp // group, N, 2)[..., 0] = 7.5      # the codes' mean
    c.x[:, :K] = c.x[:, :K].float() * deviation + mean
    c.call()
    torch.cuda.synchronize()
    assert bool((c.ws[:256] != 0xAB).any()) == in_tiles
    want, _ = c.reference()
    rel = np.linalg.norm(c.y[:, :N].double().cpu().numpy() - want) / np.linalg.norm(want)
    print(rel)
    assert rel <= shifted_tolerance(group, K, 3 if x == "fp32" else 1), rel


def test_a_workspace_serves_fewer_rows_in_tiles(torch):
    """Of the sizes here the largest T has no shares, smaller ones need up to 33 MB for theirs: the workspace of the largest has room."""
    N, K, T = 9001, 6000, 700
    c = Large(torch, T, N, K, 128, "bf16", "fp32", extra=8)
    x, y = c.x, c.y
    for c.T in (700, 600, 513, 400, 300, 200, 129, 128, 100, 64, 33):
        c.x, c.y = x[:c.T], y
        c.ws[:-64].fill_(0xAB)
        c.y.fill_(7.0)
        c.check_rows(c.T)
        assert (c.ws[:256] != 0xAB).any()


def test_two_streams_in_tiles(torch):
    """Products in tiles with shares, each with a workspace of its own, next to each other."""
    a = Large(torch, 129, 9001, 6000, 128, "bf16", "fp32", seed=1)
    b = Large(torch, 100, 6052, 3840, 32, "fp32", "fp32", seed=2)
    want = []
    for c in (a, b):
        c.check()
        assert c.in_tiles
        want.append(c.y.clone())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for c in (a, b):
        c.y.fill_(7.0)
    torch.cuda.synchronize()
    for _ in range(5):
        a.call(streams[0].cuda_stream)
        b.call(streams[1].cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(a.y, want[0]) and torch.equal(b.y, want[1])


# Products in tiles, without shares and with them, of both types of x
TILED = [(2048, 4096, 512, 128, "bf16"), (300, 2816, 4104, 64, "bf16"), (100, 6052, 3840, 32, "fp32"), (1700, 4001, 392, 64, "fp32")]
TILED_IDS = [str(c) for c in TILED]


def tiled(torch, case, **kw):
    """Behind it a workspace of NaN patterns."""
    c = Large(torch, *case, "fp32", seed=case[0], **kw)
    c.ws.fill_(0xFF)
    return c


def used(c):
    assert bool((c.ws[:256] != 0xFF).any()) and bool((c.ws[-64:] == 0xFF).all())


@pytest.mark.parametrize("case", TILED, ids=TILED_IDS)
def test_residual_in_place_in_tiles(torch, case):
    c = tiled(torch, case, bias=True, residual=True, extra=8)
    residual = c.r.clone()
    c.call()
    used(c)
    first = c.y.clone()
    c.compare()
    c.y = c.r
    c.call()
    assert torch.equal(c.r[:, :c.N], first[:, :c.N]) and torch.equal(c.r[:, c.N:], residual[:, c.N:])


@pytest.mark.parametrize("case", TILED, ids=TILED_IDS)
def test_scales_of_any_kind_in_tiles(torch, case):
    c = tiled(torch, case)
    N, K, group = c.N, c.K, c.group
    Kp = linear_w4.padded(K)
    words = c.w[N * Kp // 2:].view(torch.bfloat16).view(Kp // group, N, 2)
    z, s = words[..., 0], words[..., 1]
    s[:, 3], z[:, 3] = 0.0, 0.0
    s[1, 4] = 0.0
    s[:, 5] *= -1.0
    s[:, 6], s[:, 7] = 1e-30, 1e30
    z[:, 8], z[:, 9] = -3.625, 200.0
    s[2, 10] = float("nan")
    z[:, 11], z[:, 12] = 1e-3, 15.9375
    c.call()
    used(c)
    want, size = c.reference()
    compare(c.y.double().cpu().numpy(), want, size, group, K, c.x_type, "fp32", norm=False)
    assert (c.y[:, 3] == 0).all() and c.y[:, 10].isnan().all()


@pytest.mark.parametrize("case", TILED, ids=TILED_IDS)
def test_values_of_any_size_in_tiles(torch, case):
    c = tiled(torch, case)
    power = np.random.default_rng(1).integers(-90, 100, tuple(c.x.shape))
    c.x.copy_(c.x.double() * torch.from_numpy(2.0 ** power).cuda())
    c.call()
    used(c)
    want, size = c.reference()
    compare(c.y.double().cpu().numpy(), want, size, c.group, c.K, c.x_type, "fp32", norm=False)
    c.x.zero_()
    c.call()
    assert (c.y == 0).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("case", TILED, ids=TILED_IDS)
def test_rows_that_are_not_finite_stay_alone_in_tiles(torch, case, value):
    c = tiled(torch, case)
    c.call()
    used(c)
    clean = c.y.clone()
    bad = torch.zeros(c.T, dtype=torch.bool, device="cuda")
    bad[[0, 17, c.T - 1]] = True
    c.x[0, 5] = c.x[17, c.K - 1] = c.x[c.T - 1, c.K // 2] = value
    c.ws.fill_(0xFF)
    c.call()
    assert c.y[bad].isnan().all() and torch.equal(c.y[~bad], clean[~bad])


# T, N, K, type of x: the most that is staged in LDS whole, and 8 values more
STAGED = [(4, 700, 5760, "fp32"), (4, 700, 5768, "fp32"), (2, 333, 11520, "fp32"), (2, 333, 11528, "fp32"), (1, 700, 23168, "fp32"),
          (1, 700, 23176, "fp32"), (1, 5000, 14336, "fp32"), (4, 700, 6016, "bf16"), (4, 700, 6024, "bf16"), (1, 700, 24448, "bf16"),
          (1, 700, 24456, "bf16"), (4, 5000, 4096, "fp32")]


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("T,N,K,x", STAGED, ids=[str(c) for c in STAGED])
def test_rows_that_just_fit_into_lds(torch, T, N, K, x, group):
    print(Large(torch, T, N, K, group, x, "fp32", bias=True, residual=True, extra=8, seed=T).check())


@pytest.mark.parametrize("T", [3, 300])
def test_rows_between_others(torch, T):
    """Results between the rows of x and of the residual, in the same buffers: not refused, and right."""
    c = Large(torch, T, 264, 512, 64, "fp32", "fp32", residual=True)
    c.call()
    want = c.y.clone()
    wide = torch.cat([c.x, c.y], 1)
    c.x, c.y = wide[:, :512], wide[:, 512:]
    c.y.fill_(7.0)
    c.call()
    assert torch.equal(c.y, want)
    both = torch.cat([c.r, c.r], 1)
    c.r, c.y = both[:, 264:], both[:, :264]
    c.call()
    assert torch.equal(c.y, want) and torch.equal(c.x, wide[:, :512])
    c.r = both[:, 4:268]
    with pytest.raises(native.ApexError):
        c.call()
