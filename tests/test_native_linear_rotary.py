"""4-bit projections, rotary positions and the store with rotation on the CPU: the packer and the
frequencies against the oracle, and refusals (nothing is enqueued on these paths)."""
import numpy as np
import pytest

from oracle import linear_w4, rotary
from paper_2608_11688_amd import native

A = 4096   # a fake, aligned, never-dereferenced address
INVAL, UNSUPPORTED, CAPACITY = native.APEX_E_INVAL, native.APEX_E_UNSUPPORTED, native.APEX_E_CAPACITY
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def plan_lib():
    return native.plan_lib()


def refused(status, fn, *args, **kw):
    with pytest.raises(native.ApexError) as e:
        fn(*args, **kw)
    assert e.value.status == status, e.value


# ------------------------------------------------------------------------------ packer
def bits(w):
    return (np.asarray(w, np.float32).view(np.uint32) >> 16).astype(np.uint16)


@pytest.mark.parametrize("N,K,group", [(1, 8, 32), (3, 40, 32), (5, 128, 128), (7, 136, 64), (4, 520, 128)])
def test_packer_matches_oracle(plan_lib, N, K, group):
    rng = np.random.default_rng(N * K)
    w = rng.standard_normal((N, K)) * 10.0 ** rng.integers(-30, 30, (N, 1))
    w[0, :K // 2] = np.abs(w[0, :K // 2])              # groups of one sign: lo or hi is 0
    w[-1, K // 2:] = -np.abs(w[-1, K // 2:])
    if N > 2:
        w[1] = 0.0
        w[2, 1], w[2, 2] = 3.38e38, -3.38e38           # a range past fp32's largest
    if N > 3:
        w[3, 0], w[3, -1] = INF, NAN
    if N > 4:
        w[4] = 1e-40 * rng.integers(0, 3, K)           # subnormal, scales that round to 0 among them
    w = linear_w4.bf16(w.astype(np.float32))
    out = np.full(native.apex_linear_w4_bytes(N, K, group, L=plan_lib) + 16, 0xAB, np.uint8)
    native.apex_pack_linear_w4(bits(w), N, K, group, out, L=plan_lib)
    want = linear_w4.pack(*linear_w4.quantise(w, group))
    assert np.array_equal(out[:-16], want) and (out[-16:] == 0xAB).all()


@pytest.mark.parametrize("N,K,group", [(0, 64, 32), (-1, 64, 32), (4, 0, 32), (4, 12, 32), (4, 64, 16), (4, 64, 256),
                                       ((1 << 24) + 1, 64, 32), (4, (1 << 20) + 8, 32), (4, 64, 0)])
def test_packer_refuses(plan_lib, N, K, group):
    buf = np.zeros(64, np.uint16)
    assert native.apex_linear_w4_bytes(N, K, group, L=plan_lib) == 0
    refused(INVAL, native.apex_pack_linear_w4, buf, N, K, group, buf, L=plan_lib)


def test_packer_refuses_null(plan_lib):
    buf = np.zeros(64, np.uint16)
    refused(INVAL, native.apex_pack_linear_w4, None, 1, 8, 32, buf, L=plan_lib)
    refused(INVAL, native.apex_pack_linear_w4, buf, 1, 8, 32, None, L=plan_lib)


# ------------------------------------------------------------------------------ frequencies
@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "turns", "index"])
@pytest.mark.parametrize("dim,base,factor,original,low,high", [
    (64, 10000.0, 4.0, 4096.0, 1.0, 4.0), (128, 500000.0, 8.0, 8192.0, 1.0, 32.0), (16, 10000.0, 1.0, 100.0, 1.0, 2.0),
    (48, 1e6, 40.0, 32768.0, 1.0, 32.0), (64, 10000.0, 2.0, 1.0, 1.0, 32.0)])
def test_frequencies_match_oracle(plan_lib, scaling, dim, base, factor, original, low, high):
    got = np.full(dim // 2 + 1, 7.0)
    native.apex_rotary_frequencies(dim, base, scaling, factor, original, low, high, got, L=plan_lib)
    want = rotary.frequencies(dim, base, scaling, factor, original, low, high)
    assert np.allclose(got[:-1], want, rtol=1e-13, atol=0) and got[-1] == 7.0


@pytest.mark.parametrize("kw", [
    dict(dim=0), dict(dim=24), dict(dim=1040), dict(base=1.0), dict(base=INF), dict(base=NAN), dict(scaling=5), dict(scaling=-1),
    dict(factor=0.5), dict(factor=NAN), dict(original=0.0), dict(original=NAN), dict(low=0.0), dict(low=32.0),
    dict(high=INF), dict(freq=None), dict(scaling="base", factor=1e308, base=1e308)], ids=str)
def test_frequencies_refuse(plan_lib, kw):
    d = dict(dim=64, base=1e4, scaling="index", factor=4.0, original=4096.0, low=1.0, high=32.0, freq=np.zeros(512))
    d.update(kw)
    refused(INVAL, native.apex_rotary_frequencies, *d.values(), L=plan_lib)


def test_plain_frequencies_look_at_no_scaling(plan_lib):
    f = np.zeros(32)
    native.apex_rotary_frequencies(64, 1e4, "plain", 0.0, NAN, -1.0, -2.0, f, L=plan_lib)
    assert f[0] == 1


# ------------------------------------------------------------------------------ rotary positions
def rotate(rot=dict(), **kw):
    r = dict(layout="half", dim=64, freq=A, amplitude=1.0)
    r.update(rot)
    d = dict(x=A, dtype="bf16", T=4, heads=8, hd=128, xs=1024, pos=A, out=2 * A, os=1024)
    d.update(kw)
    native.apex_rotary(native.rotary(**r), *d.values())


BAD_ROTATIONS = [dict(layout=2), dict(layout=-1), dict(dim=0), dict(dim=8), dict(dim=24), dict(dim=144), dict(freq=None),
                 dict(freq=A + 8), dict(amplitude=INF), dict(amplitude=NAN)]


@pytest.mark.parametrize("rot", BAD_ROTATIONS, ids=str)
def test_rotations_that_are_none(rot):
    refused(INVAL, rotate, rot)
    refused(INVAL, store, rot)


def test_null_rotation():
    refused(INVAL, native.apex_rotary, None, A, "bf16", 4, 8, 128, 1024, A, 2 * A, 1024)


@pytest.mark.parametrize("status,kw", [
    (INVAL, dict(T=-1)), (UNSUPPORTED, dict(T=native.MAX_STEP_TOKENS + 1)), (INVAL, dict(dtype=2)), (INVAL, dict(heads=0)),
    (UNSUPPORTED, dict(heads=(1 << 20) + 1)), (INVAL, dict(hd=100)), (INVAL, dict(hd=8)), (UNSUPPORTED, dict(hd=1032)),
    (INVAL, dict(xs=1016)), (INVAL, dict(xs=1028)), (INVAL, dict(os=1016)), (INVAL, dict(dtype="fp32", os=1026)),
    (INVAL, dict(x=None)), (INVAL, dict(pos=None)), (INVAL, dict(out=None)), (INVAL, dict(x=A + 8)),
    (INVAL, dict(out=A + 8)), (INVAL, dict(pos=A + 2)), (INVAL, dict(out=A, os=2048))], ids=str)
def test_rotary_refuses(status, kw):
    refused(status, rotate, **kw)


# ------------------------------------------------------------------------------ store with rotation
def store(rot=dict(), cache=dict(), **kw):
    r = dict(layout="half", dim=64, freq=A, amplitude=1.0)
    r.update(rot)
    c = dict(fmt="bf16", G=8, hd=128, page_size=16, n_pages=10, k_pages=A, v_pages=A, k_scales=None, v_scales=None)
    c.update(cache)
    d = dict(q=A, k=A, v=A, dtype="bf16", T=4, H=32, qs=4096, ks=1024, vs=1024, slots=A, pos=A, out=2 * A, os=4096)
    d.update(kw)
    native.apex_paged_store_rotary(native.paged_cache(**c), native.rotary(**r), *d.values())


@pytest.mark.parametrize("status,kw", [
    (INVAL, dict(page_size=24)), (INVAL, dict(hd=96)), (INVAL, dict(fmt=2)), (INVAL, dict(k_pages=None)),
    (INVAL, dict(fmt="fp8")), (INVAL, dict(k_scales=A, v_scales=A)), (UNSUPPORTED, dict(G=1025))], ids=str)
def test_store_refuses_pools_that_are_none(status, kw):
    refused(status, store, cache=kw)


@pytest.mark.parametrize("status,kw", [
    (INVAL, dict(T=-1)), (UNSUPPORTED, dict(T=native.MAX_STEP_TOKENS + 1)), (INVAL, dict(dtype=-1)), (INVAL, dict(H=-1)),
    (UNSUPPORTED, dict(H=(1 << 20) + 1)), (INVAL, dict(qs=4088)), (INVAL, dict(qs=4100)), (INVAL, dict(ks=1016)),
    (INVAL, dict(vs=1028)), (INVAL, dict(os=4088)), (INVAL, dict(q=None)), (INVAL, dict(k=None)), (INVAL, dict(v=None)),
    (INVAL, dict(slots=None)), (INVAL, dict(pos=None)), (INVAL, dict(out=None)), (INVAL, dict(q=A + 8)),
    (INVAL, dict(k=A + 8)), (INVAL, dict(v=A + 8)), (INVAL, dict(slots=A + 2)), (INVAL, dict(pos=A + 2)),
    (INVAL, dict(out=A + 8)), (INVAL, dict(out=A, os=8192))], ids=str)
def test_store_refuses(status, kw):
    refused(status, store, **kw)


def test_null_cache_or_rotation():
    r = native.rotary("half", 64, A)
    refused(INVAL, native.apex_paged_store_rotary, None, r, A, A, A, "bf16", 1, 8, 1024, 1024, 1024, A, A, A, 1024)
    c = native.paged_cache("bf16", 8, 128, 16, 10, A, A)
    refused(INVAL, native.apex_paged_store_rotary, c, None, A, A, A, "bf16", 1, 8, 1024, 1024, 1024, A, A, A, 1024)


# ------------------------------------------------------------------------------ projection
LARGE = dict(xt="fp32", T=256, N=8192, K=8192, xs=8192, ys=8192, rs=8192)       # needs a workspace


def project(**kw):
    d = dict(w=A, N=96, K=256, group=64, x=A, xt="bf16", T=4, xs=256, bias=A, r=A, rs=96, y=2 * A, yt="bf16", ys=96,
             ws=A, n=1 << 40)
    d.update(kw)
    native.apex_linear_w4(*d.values())


@pytest.mark.parametrize("status,kw", [
    (INVAL, dict(T=-1)), (UNSUPPORTED, dict(T=native.MAX_STEP_TOKENS + 1)), (INVAL, dict(N=0)), (INVAL, dict(K=252)),
    (INVAL, dict(K=0)), (INVAL, dict(group=48)), (INVAL, dict(xt=2)), (INVAL, dict(yt=-1)), (INVAL, dict(xs=248)),
    (INVAL, dict(xs=260)), (INVAL, dict(xt="fp32", xs=258)), (INVAL, dict(ys=95)), (INVAL, dict(rs=95)),
    (INVAL, dict(w=None)), (INVAL, dict(x=None)), (INVAL, dict(y=None)), (INVAL, dict(w=A + 8)), (INVAL, dict(x=A + 8)),
    (INVAL, dict(y=A + 8)), (INVAL, dict(bias=A + 4)), (INVAL, dict(r=A + 2)), (INVAL, dict(ws=A + 8)),
    (INVAL, dict(r=2 * A, rs=200)), (INVAL, dict(y=A)), (INVAL, dict(N=(1 << 24) + 1, ys=1 << 25, rs=1 << 25)),
    (INVAL, dict(K=(1 << 20) + 8, xs=1 << 21)), (INVAL, dict(LARGE, ws=None)), (CAPACITY, dict(LARGE, n=1024)),
    (CAPACITY, dict(LARGE, xt="bf16", n=256 * 8192 * 2))], ids=str)
def test_linear_refuses(status, kw):
    refused(status, project, **kw)


def test_calls_without_work_do_nothing():
    project(T=0, w=None, x=None, y=None, ws=None, n=0)
    rotate(dict(freq=None), T=0, x=None, pos=None, out=None)
    store(T=0, q=None, k=None, v=None, slots=None, pos=None, out=None)


def test_linear_workspace():
    f = native.apex_linear_w4_workspace_bytes
    assert f(0, 96, 256, 64, "fp32") == 0 and f(4, 96, 250, 64, "fp32") == 0 and f(-1, 96, 256, 64, "bf16") == 0
    for T in (1, 100, 5000):
        assert f(T, 96, 256, 64, "fp32") <= (T + 256) * 256 * 2 * 4 + (1 << 20)
        assert f(T, 96, 256, 64, "bf16") <= (T + 256) * 256 * 2 * 2 + (1 << 20)
    assert 256 * 8192 * 6 < f(256, 8192, 8192, 64, "fp32") < (1 << 28)
    assert 256 * 8192 * 2 < f(256, 8192, 8192, 64, "bf16") < (1 << 28)
    assert f(1, 1 << 20, 1 << 20, 32, "bf16") == 0             # single rows take none
    for N, K, group, x in ((96, 256, 64, "fp32"), (4096, 4096, 32, "bf16"), (259, 3968, 128, "fp32"), (25083, 520, 64, "bf16")):
        sizes = [f(T, N, K, group, x) for T in range(1, 3000)]
        assert sizes[:16] == [0] * 16 and all(a <= b for a, b in zip(sizes, sizes[1:]))


# ------------------------------------------------------------------------------ rows that overlap
@pytest.mark.parametrize("kw", [
    dict(y=A + 16), dict(y=A + 3 * 512 + 496), dict(y=A - 48, T=1), dict(y=A - 176), dict(x=A, xs=512, y=A + 512, ys=512),
    dict(y=A + 160, ys=100), dict(r=2 * A + 16, rs=96), dict(r=2 * A - 16, rs=96), dict(r=2 * A + 64, rs=200),
    dict(r=2 * A + 176, rs=96, T=1)], ids=str)
def test_linear_refuses_rows_that_overlap(kw):
    """x: 4 bf16 rows of 512 bytes from A on; y: 4 bf16 rows of 192 bytes."""
    refused(INVAL, project, **dict(dict(y=3 * A), **({"y": 2 * A} if "r" in kw else {}), **kw))


@pytest.mark.parametrize("kw", [dict(out=A + 16), dict(out=A - 16), dict(out=A + 2048), dict(out=A + 3 * 2048 + 2032), dict(out=A + 1024, os=4096),
                                dict(xs=2048, os=2048, out=A + 2032), dict(T=1, out=A + 2032)], ids=str)
def test_rotary_refuses_rows_that_overlap(kw):
    """4 rows of 2048 bytes from A on."""
    refused(INVAL, rotate, **kw)


@pytest.mark.parametrize("kw", [dict(out=A + 16), dict(out=A + 8192), dict(k=A * 200 + 8192 - 16, out=A * 200), dict(v=A * 200 + 16, out=A * 200),
                                dict(k=A * 200 + 3 * 8192 + 8176, out=A * 200), dict(qs=6144, os=6144, out=A + 4096, q=A, k=A + 8192 + 2048)],
                         ids=str)
def test_store_refuses_rows_that_overlap(kw):
    """Queries: 4 rows of 8192 bytes from A on; keys and values: of 2048."""
    refused(INVAL, store, **dict(dict(k=A * 100, v=A * 150), **kw))
