"""PagedCache hands every page to one conversation at a time, and takes all of a step's pages or none."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2510_25600_b200.paged import PagedCache


def cache(n_pages=10, page=4, requests=3, max_rows=30):
    return PagedCache(2, n_pages, page, 1, 64, torch.bfloat16, requests, max_rows, device="cpu")


def consistent(c):
    held = [p for pages in c._pages for p in pages]
    assert sorted(held + c._free) == list(range(c.n_pages))
    for r, pages in enumerate(c._pages):
        assert len(pages) == -(-c.h_lens[r] // c.page_size) and c.block_table[r, :len(pages)].tolist() == pages
    assert c.seq_lens.tolist() == c.h_lens.tolist()


def test_rows_come_and_go():
    c = cache()
    c.set_rows([5, 0, 4])
    consistent(c)
    assert c.free_pages == 7
    first = list(c._pages[0])
    c.advance()                      # the two that have rows
    consistent(c)
    assert c.h_lens.tolist() == [6, 0, 5] and c._pages[0] == first and c.free_pages == 6
    c.advance([3, 8])
    consistent(c)
    c.advance(np.int64(0))
    consistent(c)
    assert c.h_lens.tolist() == [9, 8, 5]
    c.release(0)
    consistent(c)
    assert c.h_lens.tolist() == [0, 8, 5] and c.free_pages == 6
    c.set_rows([24])
    consistent(c)
    assert c.free_pages == 0


def test_all_or_nothing():
    c = cache()
    c.set_rows([20, 8, 0])
    before = [list(p) for p in c._pages], c.h_lens.tolist(), list(c._free)
    with pytest.raises(RuntimeError):
        c.set_rows([24, 8, 13])
    with pytest.raises(ValueError):
        c.set_rows([31])
    with pytest.raises(ValueError):
        c.set_rows([-1])
    with pytest.raises(ValueError):
        c.set_rows([1, 1, 1, 1])
    assert before == ([list(p) for p in c._pages], c.h_lens.tolist(), list(c._free))
    consistent(c)
    c.set_rows([4, 8, 16])           # pages given back in the same step are there to be taken
    consistent(c)


def test_a_refused_prompt_takes_no_rows():
    c = cache()
    c.set_rows([5, 0, 4])
    before = c.h_lens.tolist(), c.free_pages
    ints = lambda *x: torch.tensor(x, dtype=torch.int32)
    batch = SimpleNamespace(n_req=2, cu_seqlens=ints(0, 6, 12))
    budget = SimpleNamespace(h_cu_kept=np.array([0, 3, 7]), cu_kept=ints(0, 3, 7))
    k = torch.zeros((2, 12, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # not on a GPU
        c.store_prompt(k, k, torch.zeros((2, 1, 7), dtype=torch.int32), batch, budget)
    assert before == (c.h_lens.tolist(), c.free_pages)
    consistent(c)


def test_random_steps():
    rng = np.random.default_rng(0)
    c = cache(40, 3, 6, 60)
    for _ in range(300):
        rows = rng.integers(0, 30, size=rng.integers(1, 7))
        try:
            c.set_rows(rows)
        except RuntimeError:
            c.release(int(rng.integers(0, 6)))
        consistent(c)


def test_sizes():
    with pytest.raises(ValueError):
        cache(n_pages=0)
    assert cache(page=7, max_rows=15).max_pages == 3
