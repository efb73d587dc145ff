"""Pins of the paged-cache oracle: a worked plan, the window's definition, attention over one
page against plain attention, and invariants of random plans."""
import numpy as np
import pytest

from oracle import attention as oatt
from oracle import paged


def test_plan_worked_example():
    # page 16; request 0 holds 16 positions (page 7) and wants 2, request 1 ends and gives back
    # pages 3 and 9, request 2 is new with 33 tokens, request 3 wants more than is left
    table = np.array([[7, -1, -1], [3, 9, -1], [-1, -1, -1], [-1, -1, -1]])
    r = paged.plan([16, 20, 0, 0], [2, -1, 33, 40], 16, 10, table, 64, [5, 4, 0, 0, 0, 0, 0, 0, 0, 0], 2)
    # stack: 5 4 | 3 9; taken from the top: 9 for request 0, then 3, 4, 5 for request 2
    assert r["block_table"].tolist() == [[7, 9, -1], [3, 9, -1], [3, 4, 5], [-1, -1, -1]]
    assert r["free_count"] == 0 and r["free_pages"][:4].tolist() == [5, 4, 3, 9]
    assert r["status"].tolist() == [paged.SERVED, paged.ENDED, paged.SERVED, paged.WAITS]
    assert r["seq_len"].tolist() == [18, 0, 33, 0] and r["cu_new"].tolist() == [0, 2, 2, 35, 35]
    assert r["slot_map"][:3].tolist() == [9 * 16, 9 * 16 + 1, 3 * 16] and r["slot_map"][34] == 5 * 16
    assert (r["slot_map"][35:] == -1).all() and r["positions"][:3].tolist() == [16, 17, 0]


@pytest.mark.parametrize("seed", range(6))
def test_plan_never_hands_out_a_page_twice(seed):
    rng = np.random.default_rng(seed)
    R, page, width, n_pages = 12, 16, 9, 60
    table, cached = np.full((R, width), -1), np.zeros(R, np.int64)
    free, count = np.arange(n_pages), n_pages
    for _ in range(25):
        n_new = rng.integers(-1, 40, R)
        r = paged.plan(cached, n_new, page, n_pages, table, 150, free, count)
        table, cached, free, count = r["block_table"], r["seq_len"], r["free_pages"], r["free_count"]
        held = [table[q, b] for q in range(R) for b in range(-(-int(cached[q]) // page))]
        assert sorted(held + list(free[:count])) == list(range(n_pages))
        assert r["cu_new"][-1] <= 150


def test_visible_positions():
    assert paged.visible_positions(3, 0, 0).tolist() == [0, 1, 2, 3]
    assert paged.visible_positions(9, 3, 2).tolist() == [0, 1, 7, 8, 9]
    assert paged.visible_positions(2, 3, 9).tolist() == [0, 1, 2]
    assert paged.visible_positions(5, 1, 0).tolist() == [5]


def test_attention_over_scattered_pages_equals_plain_attention():
    rng = np.random.default_rng(1)
    H, G, hd, page = 4, 2, 8, 16
    K, V = rng.standard_normal((2, 40, G, hd))
    pages = rng.standard_normal((2, 5, G, page, hd))
    order = [4, 0, 2]
    for j in range(40):
        pages[0, order[j // page], :, j % page], pages[1, order[j // page], :, j % page] = K[j], V[j]
    q = rng.standard_normal((2, H, hd))
    got, size, _ = paged.attend(q, pages[0], pages[1], [0, 2], [40], np.array([order]), 0, 0, 0.3, np.zeros_like(q))
    for i, p in enumerate((38, 39)):
        for h in range(H):
            want = oatt.attend(q[i, h], K[:p + 1, h // 2], V[:p + 1, h // 2], 0.3)
            assert np.allclose(got[i, h], want, rtol=1e-13, atol=1e-15)
    assert (size >= np.abs(got)).all()


def test_a_row_that_sees_nothing_is_zero_and_rows_behind_stay():
    q = np.ones((3, 1, 4))
    pages = np.ones((2, 1, 16, 4))
    out, _, _ = paged.attend(q, pages, pages, [0, 1, 2], [3, 0], np.array([[-1], [0]]), 0, 0, 1.0, np.full((3, 1, 4), 7.0))
    assert (out[0] == 0).all() and (out[1] == 0).all() and (out[2] == 7).all()


def test_a_row_whose_scores_are_all_minus_infinity_is_zero():
    q = np.array([[[1.0, 2.0]], [[-1.0, 0.5]]])
    pages = np.ones((2, 1, 1, 16, 2))
    pages[0, 0, 0, :2, 0] = -np.inf
    with np.errstate(invalid="ignore"):
        out, size, _ = paged.attend(q, pages[0], pages[1], [0, 1, 2], [2, 1], np.array([[0], [0]]), 0, 0, 1.0,
                                    np.full((2, 1, 2), 7.0))
    assert (out[0] == 0).all() and (size[0] == 0).all()
    assert np.isnan(out[1]).all()                   # a score of +infinity


def test_store_rounds_rows():
    rows = np.array([[[1.0, -448.0, 2.0 ** -9, 0.0]], [[np.inf, 1, 1, 1]], [[0.0, 0, 0, 0]]])
    codes, scales = np.zeros((1, 1, 16, 4), np.uint8), np.full((1, 1, 16), 9.0, np.float32)
    paged.store(rows, [3, 4, 5], 16, codes, scales)
    assert codes[0, 0, 3].tolist() == [0x38, 0xFE, 0x01, 0x00] and scales[0, 0, 3] == 1.0
    assert np.isnan(scales[0, 0, 4]) and scales[0, 0, 5] == 0 and scales[0, 0, 6] == 9
    pages = np.zeros((1, 1, 16, 4))
    paged.store(np.array([[[1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 0, -1]]]), [16], 16, pages, None)
    assert (pages == 0).all()                      # slot out of range
    paged.store(np.array([[[1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 0, -1]]]), [2], 16, pages, None)
    assert pages[0, 0, 2].tolist() == [1.0, 1 + 2.0 ** -6, 0.0, -1.0]
