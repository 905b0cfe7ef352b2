"""GPU: powattn_page_tables against the tokens taken one after the other.  Whole numbers: equal."""
import numpy as np
import pytest
import torch

from around_util import tables
from paper_2503_03588_amd import binding as pa

pytestmark = pytest.mark.gpu


def check(block, stride, q_start, q_len, q_rows, n_free, n_pages, seed, holes=False):
    rng = np.random.default_rng(seed)
    batch = len(q_start)
    table = rng.permutation(batch * stride).reshape(batch, stride) % n_pages
    if holes:
        table[rng.random(table.shape) < 0.3] = -1
        table[rng.random(table.shape) < 0.1] = n_pages
    free = rng.permutation(max(n_free, 1))[:n_free] + 1000
    want = tables(block, q_start, q_len, q_rows, free, n_pages, table)
    dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    d_table, d_free = dev(table), dev(free.reshape(-1))
    for _ in range(2):                                     # the same lengths again give the same pages
        slots, kv_len, taken = pa.page_tables(pa.Pattern(block, 4, 1), dev(q_start), dev(q_len), d_free, d_table, n_pages, q_rows)
        for got, exact in zip((d_table, slots, kv_len, taken), want):
            assert np.array_equal(got.cpu().numpy(), np.asarray(exact).reshape(got.shape))


@pytest.mark.parametrize("block", [64, 128, 48, 1])
@pytest.mark.parametrize("batch", [1, 5, 256, 257, 700])
def test_one_token_each(block, batch):
    rng = np.random.default_rng(batch)
    start = rng.integers(0, 8 * block, size=batch)
    start[: batch // 3] -= start[: batch // 3] % block     # a page for every third sequence at least
    check(block, 8, start, np.ones(batch, int), 1, batch + 5, 10 ** 4, seed=1)


@pytest.mark.parametrize("q_rows", [2, 3, 100, 128, 129, 256, 257, 1024, 1025, 3000])
def test_ragged_pieces(q_rows):
    rng = np.random.default_rng(q_rows)
    batch = 37
    start, n = rng.integers(0, 5000, size=batch), rng.integers(0, q_rows + 1, size=batch)
    n[3], n[5], start[7] = 0, q_rows, 0
    check(64, 160, start, n, q_rows, 4000, 10 ** 5, seed=2)


def test_lengths_outside_the_table_and_a_list_that_is_too_short():
    start, n = np.array([-5, 0, 630, 640, 9000, 100, 64]), np.array([70, -3, 200, 5, 5, 1000, 64])
    for n_free in (0, 1, 2, 3, 50):
        check(64, 10, start, n, 300, n_free, 10 ** 5, seed=3)


def test_pages_that_are_not_there():
    rng = np.random.default_rng(4)
    check(64, 20, rng.integers(0, 1200, size=50), rng.integers(0, 80, size=50), 80, 40, 1020, seed=4, holes=True)


def test_many_sequences_and_long_pieces():
    rng = np.random.default_rng(5)
    check(64, 4, rng.integers(0, 200, size=3001), rng.integers(0, 6, size=3001), 5, 9000, 10 ** 6, seed=5)
    check(64, 900, [17], [50001], 50001, 1000, 10 ** 6, seed=6)


def test_outputs_given_and_rows_of_other_sequences_untouched():
    pat = pa.Pattern(64, 4, 1)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.full((2, 5), 77, dtype=torch.int32, device="cuda")
    slots, kv_len, taken = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), i32(0, 0), i32(0)
    out = pa.page_tables(pat, i32(63, 128), i32(2, 0), i32(5, 6), table, 100, 3, slots=slots, kv_len=kv_len, n_taken=taken)
    assert out[0] is slots and out[1] is kv_len and out[2] is taken
    assert slots.tolist() == [[77 * 64 + 63, 5 * 64, -1], [-1] * 3] and kv_len.tolist() == [65, 128] and taken.tolist() == [1]
    assert table.tolist() == [[77, 5, 77, 77, 77], [77] * 5]
