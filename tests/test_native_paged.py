"""Refusals of the paged-cache entry points (CPU only: nothing is enqueued on these paths)."""
import pytest

from paper_2608_11688_amd import native

A = 4096   # a fake, aligned, never-dereferenced address


def refused(status, fn, *args):
    with pytest.raises(native.ApexError) as e:
        fn(*args)
    assert e.value.status == status, e.value


def cache(fmt="bf16", G=8, hd=128, page=16, n_pages=10, k=A, v=A, ks=None, vs=None):
    return native.paged_cache(fmt, G, hd, page, n_pages, k, v, ks, vs)


INVAL, UNSUPPORTED, CAPACITY = native.APEX_E_INVAL, native.APEX_E_UNSUPPORTED, native.APEX_E_CAPACITY

BAD_CACHES = [
    (INVAL, dict(page=24)), (INVAL, dict(page=8)), (INVAL, dict(page=2048)), (INVAL, dict(n_pages=0)),
    (INVAL, dict(hd=96)), (INVAL, dict(G=0)), (INVAL, dict(fmt=2)), (INVAL, dict(k=None)), (INVAL, dict(v=None)),
    (INVAL, dict(k=A + 8)), (INVAL, dict(v=A + 2)), (INVAL, dict(fmt="fp8")), (INVAL, dict(fmt="fp8", ks=A)),
    (INVAL, dict(fmt="fp8", ks=A, vs=A + 4)), (INVAL, dict(ks=A, vs=A)), (UNSUPPORTED, dict(G=1025)),
    (UNSUPPORTED, dict(page=1024, n_pages=1 << 21)),
]


def store(c, **kw):
    d = dict(k=A, v=A, dtype="bf16", T=4, ks=1024, vs=1024, slots=A)
    d.update(kw)
    native.apex_paged_store(c, d["k"], d["v"], d["dtype"], d["T"], d["ks"], d["vs"], d["slots"])


def attend(c, **kw):
    d = dict(q=A, dtype="bf16", T=4, R=2, H=32, qs=4096, cu=A, seq=A, table=A, nb=4, window=0, sinks=0,
             scale=0.1, out=A, os=4096, ws=A, n=1 << 40)
    d.update(kw)
    native.apex_attention_paged(c, d["q"], d["dtype"], d["T"], d["R"], d["H"], d["qs"], d["cu"], d["seq"],
                                d["table"], d["nb"], d["window"], d["sinks"], d["scale"], d["out"], d["os"],
                                d["ws"], d["n"])


@pytest.mark.parametrize("status,kw", BAD_CACHES, ids=[str(sorted(c[1].items())) for c in BAD_CACHES])
def test_pools_that_are_none(status, kw):
    refused(status, store, cache(**kw))
    refused(status, attend, cache(**kw))


def test_null_cache():
    refused(INVAL, store, None)
    refused(INVAL, attend, None)


@pytest.mark.parametrize("kw", [dict(T=-1), dict(dtype=2), dict(ks=1016), dict(vs=1016), dict(ks=1028), dict(k=None),
                                dict(v=None), dict(slots=None), dict(k=A + 8), dict(v=A + 8), dict(slots=A + 2),
                                dict(dtype="fp32", ks=1026)], ids=str)
def test_store_refuses(kw):
    refused(INVAL, lambda: store(cache(), **kw))


def test_store_of_more_rows_than_a_grid_has():
    refused(UNSUPPORTED, lambda: store(cache(G=1024), T=2 ** 31 - 1, ks=1024 * 128, vs=1024 * 128))


@pytest.mark.parametrize("status,kw", [
    (INVAL, dict(T=-1)), (INVAL, dict(R=-1)), (INVAL, dict(dtype=-1)), (INVAL, dict(H=20)), (INVAL, dict(H=0)),
    (UNSUPPORTED, dict(H=136, qs=136 * 128, os=136 * 128)), (UNSUPPORTED, dict(R=native.MAX_REQUESTS + 1)),
    (UNSUPPORTED, dict(T=native.MAX_STEP_TOKENS + 1)), (INVAL, dict(nb=0)), (UNSUPPORTED, dict(nb=1 << 27)),
    (INVAL, dict(window=-1)), (INVAL, dict(sinks=-1)),
    (INVAL, dict(scale=0.0)), (INVAL, dict(scale=float("inf"))), (INVAL, dict(scale=float("nan"))),
    (INVAL, dict(scale=-1.0)), (INVAL, dict(qs=4088)), (INVAL, dict(os=4088)), (INVAL, dict(qs=4100)),
    (INVAL, dict(q=None)), (INVAL, dict(out=None)), (INVAL, dict(cu=None)), (INVAL, dict(seq=None)),
    (INVAL, dict(table=None)), (INVAL, dict(ws=None)), (INVAL, dict(q=A + 8)), (INVAL, dict(out=A + 8)),
    (INVAL, dict(ws=A + 8)), (INVAL, dict(table=A + 2)), (CAPACITY, dict(n=1024)),
], ids=str)
def test_attention_refuses(status, kw):
    refused(status, lambda: attend(cache(), **kw))


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_scales_whose_powers_of_two_are_infinite(scale):
    refused(INVAL, lambda: attend(cache(), scale=scale))


def plan(**kw):
    names = ("cached", "n_new", "free", "count", "table", "seq", "cu", "slots", "pos", "count_out", "status")
    d = dict(R=3, page=16, n_pages=10, nb=4, T=8, **{n: A * (i + 1) for i, n in enumerate(names)})
    d.update(kw)
    native.apex_paged_plan(d["cached"], d["n_new"], d["R"], d["page"], d["n_pages"], d["nb"], d["T"], d["free"],
                           d["count"], d["table"], d["seq"], d["cu"], d["slots"], d["pos"], d["count_out"], d["status"])


@pytest.mark.parametrize("status,kw", [
    (INVAL, dict(R=-1)), (UNSUPPORTED, dict(R=native.MAX_REQUESTS + 1)), (INVAL, dict(page=20)), (INVAL, dict(n_pages=0)),
    (UNSUPPORTED, dict(n_pages=1 << 27)), (INVAL, dict(nb=0)), (UNSUPPORTED, dict(nb=1 << 27)), (INVAL, dict(T=-1)),
    (INVAL, dict(cached=None)), (INVAL, dict(n_new=None)), (INVAL, dict(free=None)), (INVAL, dict(count=None)),
    (INVAL, dict(table=None)), (INVAL, dict(seq=None)), (INVAL, dict(cu=None)), (INVAL, dict(slots=None)),
    (INVAL, dict(count_out=None)), (INVAL, dict(cached=A + 2)),
    (INVAL, dict(seq=A)),                  # in place of `cached`, which other workgroups still read
    (INVAL, dict(count_out=4 * A)),        # in place of free_count
], ids=str)
def test_plan_refuses(status, kw):
    refused(status, lambda: plan(**kw))


NAMES = ("cached", "n_new", "count", "free", "table", "seq", "cu", "slots", "pos", "count_out", "status")


@pytest.mark.parametrize("i,j", [(i, j) for i in range(3, len(NAMES)) for j in range(i)],
                         ids=lambda x: NAMES[x])
def test_plan_refuses_an_output_in_place_of_another_argument(i, j):
    refused(INVAL, lambda: plan(**{NAMES[i]: 64 * A, NAMES[j]: 64 * A}))


def test_calls_without_work_do_nothing():
    store(cache(), T=0, k=None, v=None, slots=None)
    attend(cache(), T=0, q=None, out=None, ws=None, n=0)
    attend(cache(), R=0, q=None, out=None, ws=None, n=0)


def test_workspace_does_not_grow_with_the_context():
    f = native.apex_attention_paged_workspace_bytes
    assert f(1, 1, 32, 8, 128) < 20 << 20 and f(4096, 8, 32, 8, 128) < 72 << 20
    assert f(0, 0, 32, 8, 128) == 256
    assert f(2 ** 31 - 1, 2 ** 31 - 1, 16, 1, 128) < 80 << 20
