"""Pools at the sizes where a call takes another path, and entries that are no pages, against the plain model of a pool."""
import numpy as np
import pytest
import torch

from test_gpu_pages import END, Model, count_refs, i32, load, pooled, same

pytestmark = pytest.mark.gpu


def test_a_fork_copies_entries_that_are_no_pages_as_none():
    """Of a parent's full pages and of its partly filled one."""
    eng = pooled(60, 4, 6, 2, 64, 2)
    load(eng, [70, 7, 50, 3])      # 69 cached: entries 0 to 3 full, entry 4 in part; 49: 0 to 2, and 3
    eng.reserve(1, i32([0] * 4))
    for b, i, bad in ((0, 1, -5), (0, 3, 60), (2, 0, 2 ** 31 - 1), (2, 3, -2 ** 31)):
        eng.page_refs[eng.block_table[b, i].item()] -= 1
        eng.block_table[b, i] = bad
    m = Model(eng)
    parent = np.asarray([0, 0, 2, 2])
    eng.fork(i32(parent)), m.fork(parent)
    for b in (1, 3):
        m.table[b][(m.table[b] < 0) | (m.table[b] >= 60)] = -1
    same(eng, m)
    assert eng.block_table[1, :5].tolist()[1::2] == [-1, -1] and (eng.block_table[3, [0, 3]] == -1).all()
    assert (count_refs(eng) == m.refs).all()
    eng.close()


@pytest.mark.parametrize("pages", [16383, 16384, 16385, 16448])
def test_pools_around_the_largest_small_one(pages):
    """Up to 16384 pages one workgroup has the index in LDS."""
    eng = pooled(pages, 6, 40, seed=pages)
    rng = np.random.default_rng(pages)
    load(eng, [int(x) for x in rng.integers(1, 600, 6)])
    m = Model(eng)
    held = rng.random(pages) < 0.7
    held[-1] = False
    held[:16300] |= rng.random(16300) < 0.995      # (the free ones lie at the end)
    eng.page_refs.copy_(i32(held))
    m.refs[:] = held
    for extra in (1, 48, 500):
        eng.reserve(extra), m.reserve(extra)
        same(eng, m, extra)
    eng.fork(i32([0, 0, 2, 2, 4, 4])), m.fork(np.asarray([0, 0, 2, 2, 4, 4]))
    same(eng, m)
    live, to = m.compact()
    assert eng.compact().item() == live
    same(eng, m)
    eng.reserve(600), m.reserve(600)
    same(eng, m)
    eng.close()


@pytest.mark.parametrize("pages", [900, 17000])
@pytest.mark.parametrize("extra", [32, 33, 47, 48, 49, 64])
def test_reservations_around_the_largest_small_one(extra, pages):
    """Up to 48 positions more a thread looks at a sequence's entries; they begin anywhere in a page."""
    eng = pooled(pages, 17, 12)
    load(eng, list(range(15, 32)), [50] * 16 + [0])
    m = Model(eng)
    eng.reserve(extra), m.reserve(extra)
    same(eng, m)
    eng.free_pages(i32([16] * 17), i32([48] * 17)), m.free([16] * 17, [48] * 17)
    eng.reserve(extra), m.reserve(extra)
    same(eng, m)
    eng.close()


@pytest.mark.parametrize("batch", [1023, 1024, 1025])
def test_batches_around_the_largest_small_one(batch):
    """Up to 1024 sequences a workgroup has a thread for each."""
    eng = pooled(6000, batch, 6)
    rng = np.random.default_rng(batch)
    load(eng, [int(x) for x in rng.integers(0, 90, batch)])
    m = Model(eng)
    for extra in (1, 20, 48, 60):
        eng.reserve(extra), m.reserve(extra)
        same(eng, m, extra)
    parent = rng.integers(-1, batch, batch)
    eng.fork(i32(parent)), m.fork(parent)
    same(eng, m)
    eng.free_pages(i32([0] * batch), i32([END] * batch))
    assert eng.compact().item() == 0 and (eng.page_refs == 0).all()
    eng.close()


def test_forks_in_a_large_pool():
    """More pages than 64 times 4096, the free ones far apart and behind the first 262144: every child's copy is the r-th free page."""
    pages, B = 270001, 40
    eng = pooled(pages, B, 8)
    load(eng, [100] * B)
    held = np.ones(pages, np.int32)
    free = np.concatenate([[3, 4095, 4096, 70000, 200000, 262143, 262144], np.arange(262150, 270001, 397)])
    held[free] = 0
    eng.block_table[0, :7] = i32([10, 11, 12, 13, 14, 15, 269999])
    eng.page_refs.copy_(i32(held))
    kc, vc = eng.kc.view(pages, -1), eng.vc.view(pages, -1)
    want = kc[269999].clone(), vc[269999].clone()
    eng.fork(i32([0] * B))
    torch.cuda.synchronize()
    table = eng.block_table.cpu().numpy()
    n = min(B - 1, len(free))
    full = n + 1 < B
    assert (table[1:n + 1, :6] == np.arange(10, 16)).all() and (table[1:n + 1, 6] == free[:n]).all() and (table[1:n + 1, 7] == -1).all()
    assert (table[n + 1:] == -1).all() and eng.poll_error() == (8 if full else 0)
    at = torch.as_tensor(free[:n], device="cuda:0")
    assert (kc[at] == want[0]).all() and (vc[at] == want[1]).all()
    refs = held.copy()
    refs[10:16] += n
    refs[free[:n]] = 1
    assert (eng.page_refs.cpu().numpy() == refs).all()
    eng.close()
