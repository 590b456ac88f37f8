"""The cache's pages against a plain model of them: tables, references, lengths and the cache's bits, which all have to be equal."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
END = 2 ** 31 - 1
EXHAUSTED, REFUSED = 8, 16


def pooled(pages, batch, width, hkv=1, hd=64, layers=1, precise=False, w_max=4, seed=0):
    from types import SimpleNamespace
    from paper_2508_18588_amd.runtime import Engine
    d = f = 64
    sh = SimpleNamespace(d_model=d, n_q_heads=hkv, n_kv_heads=hkv, head_dim=hd, d_ffn=f, vocab=512, rms_eps=1e-6)
    mat = lambda r, c: torch.zeros(r, c, device="cuda:0", dtype=torch.bfloat16)
    head, ones = mat(512, d), torch.ones(d, device="cuda:0")
    w = {"embed": head, "lm_head": head, "norm_f": ones, "wqkv": [mat(3 * hkv * hd, d)] * layers, "wo": [mat(d, hkv * hd)] * layers,
         "wgate": [mat(f, d)] * layers, "wup": [mat(f, d)] * layers, "wdown": [mat(d, f)] * layers, "norm1": [ones] * layers, "norm2": [ones] * layers}
    eng = Engine(sh, w, torch.zeros(16 * width + 64, hd // 2, 2, device="cuda:0"), max_batch=batch, k_max=0, c_max=1, max_len=16 * width - 1,
                 w_max=w_max, keep_logits=False, precise=precise, pages=pages)
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    for t in (eng.kc, eng.vc):
        t.copy_(torch.randint(-30000, 30000, t.shape, generator=g, device="cuda:0").to(t.dtype))
    return eng


class Model:
    """The same pool in numpy."""

    def __init__(self, eng):
        self.table, self.refs = eng.block_table.cpu().numpy().copy(), eng.page_refs.cpu().numpy().copy()
        self.layers, self.pages = eng.n_layers, eng.n_blocks
        self.k = eng.kc.cpu().numpy().reshape(self.layers, self.pages, -1).copy()
        self.v = eng.vc.cpu().numpy().reshape(self.layers, self.pages, -1).copy()
        self.batch = eng.batch
        self.state = {n: getattr(eng, n).cpu().numpy().copy() for n in ("seq_len", "tail", "tail_len", "k_state", "budget_left", "tokens")}
        self.seq_id = eng.seq_id.cpu().numpy().copy()
        self.error = 0

    def page(self, p):
        return 0 <= p < self.pages

    def drop(self, p):
        if not self.page(p):
            return
        if self.refs[p] <= 0:
            self.error |= REFUSED
        else:
            self.refs[p] -= 1

    def free(self, first, end):
        for b in range(self.batch):
            for i in range(self.table.shape[1]):
                if 16 * i >= first[b] and 16 * i + 16 <= end[b]:
                    self.drop(self.table[b, i])
                    self.table[b, i] = -1

    def fork(self, parent):
        pool, o, n = [int(p) for p in np.nonzero(self.refs == 0)[0]], 0, self.state["seq_len"]
        width, todo = self.table.shape[1], []
        for b in range(self.batch):
            p = int(parent[b])
            if p < 0 or p == b:
                continue
            if p >= self.batch or (parent[p] >= 0 and parent[p] != p) or n[p] < 1 or (n[p] + 14) // 16 > width:
                self.error |= REFUSED
                continue
            full, row = (int(n[p]) - 1) // 16, np.full(width, -1, np.int32)
            row[:full] = self.table[p, :full]
            if (n[p] - 1) % 16 and self.page(self.table[p, full]):
                if o == len(pool):
                    self.error |= EXHAUSTED
                    continue
                row[full] = pool[o]
                for t in (self.k, self.v):
                    t[:, pool[o]] = t[:, self.table[p, full]]
                o += 1
            todo.append((b, p, row))
        for b, p, row in todo:
            for i in range(width):
                if self.page(row[i]):
                    self.refs[row[i]] += 1
            old = self.table[b].copy()
            self.table[b] = row
            for i in range(width):
                self.drop(old[i])
            for name in ("tail", "tail_len", "k_state", "budget_left"):
                self.state[name][b] = self.state[name][p]
            self.state["tokens"][b, :n[p]] = self.state["tokens"][p, :n[p]]
        for b, p, row in todo:
            n[b] = n[p]

    def reserve(self, extra, first=None):
        pool, o, n = [int(p) for p in np.nonzero(self.refs == 0)[0]], 0, self.state["seq_len"]
        for b in range(self.batch):
            if n[b] < 1 or self.state["budget_left"][b] <= 0:
                continue
            L = int(n[b]) - 1
            for i in range((L if first is None else max(0, int(first[b]))) // 16, min(self.table.shape[1], (L + extra + 15) // 16)):
                if self.page(self.table[b, i]):
                    continue
                self.table[b, i] = -1
                if o == len(pool):
                    self.error |= EXHAUSTED
                    continue
                self.table[b, i] = pool[o]
                self.refs[pool[o]] = 1
                o += 1

    def compact(self):
        held = self.refs != 0
        live = int(held.sum())
        to = np.where(held, np.arange(self.pages), -1)
        src, dst = np.nonzero(held[live:])[0] + live, np.nonzero(~held[:live])[0]
        to[src] = dst
        for t in (self.k, self.v):
            t[:, dst] = t[:, src]
        self.refs[dst], self.refs[src] = self.refs[src], 0
        ok = (self.table >= 0) & (self.table < self.pages)
        new = to[np.where(ok, self.table, 0)]
        self.table = np.where(ok & (new >= 0), new, self.table).astype(np.int32)
        return live, to


def same(eng, m, what=""):
    torch.cuda.synchronize()
    assert eng.poll_error() == m.error, what
    m.error = 0
    assert (eng.block_table.cpu().numpy() == m.table).all(), what
    assert (eng.page_refs.cpu().numpy() == m.refs).all(), what
    for name, want in m.state.items():
        assert (getattr(eng, name).cpu().numpy() == want).all(), (what, name)
    assert (eng.seq_id.cpu().numpy() == m.seq_id).all()
    assert (eng.kc.cpu().numpy().reshape(m.k.shape) == m.k).all() and (eng.vc.cpu().numpy().reshape(m.v.shape) == m.v).all(), what


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda:0")


def load(eng, lens, budgets=None, seed=1):
    rng = np.random.default_rng(seed)
    eng.load_sequences([rng.integers(0, 512, n).astype(np.int32) for n in lens], [50] * len(lens) if budgets is None else budgets,
                       seq_ids=1000 + np.arange(eng.max_batch))


def count_refs(eng):
    """References that follow from the tables alone."""
    t = eng.block_table.cpu().numpy().reshape(-1)
    return np.bincount(t[(t >= 0) & (t < eng.n_blocks)], minlength=eng.n_blocks)


@pytest.mark.parametrize("hkv,hd,layers,precise", [(1, 64, 1, False), (3, 128, 2, False), (4, 64, 5, False), (2, 64, 2, True)])
def test_a_life_of_pages(hkv, hd, layers, precise):
    """Reserve, fork, free and compact in any order, with sequences that end, take other texts and outgrow what is left."""
    eng = pooled(90, 9, 12, hkv, hd, layers, precise, seed=layers)
    rng = np.random.default_rng(layers)
    load(eng, [int(x) for x in rng.integers(1, 150, 9)], [50, 0, 50, 50, 9, 50, 1, 50, 50])
    m = Model(eng)
    for step in range(40):
        op = ["reserve", "fork", "free", "compact", "reserve"][step % 5] if step < 10 else rng.choice(["reserve", "fork", "free", "compact"])
        if op == "reserve":
            extra = int(rng.choice([0, 1, 5, 16, 17, 60, 10 ** 9]))
            first = rng.integers(-40, 200, 9) if rng.random() < 0.3 else None
            eng.reserve(extra, None if first is None else i32(first))
            m.reserve(extra, first)
        elif op == "fork":
            parent = rng.integers(-2, 11, 9)
            eng.fork(i32(parent))
            m.fork(parent)
        elif op == "free":
            first, end = rng.integers(-20, 200, 9), rng.integers(-20, 250, 9)
            end[rng.random(9) < 0.3] = END
            eng.free_pages(i32(first), i32(end))
            m.free(first, end)
        else:
            moved = torch.full((90,), -7, dtype=torch.int32, device="cuda:0")
            live, to = m.compact()
            assert eng.compact(moved).item() == live
            assert (moved.cpu().numpy() == to).all()
        same(eng, m, (step, op))
        assert (count_refs(eng) == m.refs).all()
        if step % 7 == 6:      # texts grow and shrink between calls
            m.state["seq_len"][:] = rng.integers(0, 180, 9)
            eng.seq_len.copy_(i32(m.state["seq_len"]))
    eng.close()


def test_forks_of_every_rest():
    for n in list(range(1, 36)) + [191, 192]:
        eng = pooled(64, 4, 12, 2, 64, 2, seed=n)
        load(eng, [n, 7, 100, 3])
        m = Model(eng)
        eng.reserve(1), m.reserve(1)
        same(eng, m, n)
        eng.fork(i32([0, 0, -1, 0])), m.fork(np.asarray([0, 0, -1, 0]))
        same(eng, m, n)
        eng.close()


def test_what_a_fork_refuses():
    """A parent that takes another text itself, one outside the batch, one without tokens, one that has outgrown its table; the others go on."""
    eng = pooled(64, 8, 4, 1, 64, 1)
    load(eng, [40, 10, 20, 0, 30, 33, 17, 18])
    eng.seq_len[4] = 66      # 65 cached tokens in a table for 64
    m = Model(eng)
    for parent in ([1, 0, 2, 2, 4, 4, 8, 0], [0, 0, 1, 3, 4, 3, 2 ** 31 - 1, -2 ** 31], [0, 0, 0, 0, 0, 0, 0, 0], [5, 5, 5, 5, 5, 5, 5, 5]):
        eng.reserve(16), m.reserve(16)
        eng.fork(i32(parent)), m.fork(np.asarray(parent))
        same(eng, m, parent)
    eng.seq_len[2] = 65      # exactly full: 64 cached tokens
    m.state["seq_len"][2] = 65
    eng.fork(i32([2, 2, 2, -1, -1, -1, -1, -1])), m.fork(np.asarray([2, 2, 2, -1, -1, -1, -1, -1]))
    same(eng, m)
    eng.close()


def test_no_page_is_left():
    eng = pooled(7, 5, 6, 1, 64, 2)
    load(eng, [40, 20, 20, 20, 50])
    m = Model(eng)
    eng.reserve(1), m.reserve(1)
    same(eng, m)
    eng.free_pages(i32([0] * 5), i32([END] * 5)), m.free([0] * 5, [END] * 5)
    for b, n in ((0, 3), (4, 2)):
        m.table[b, :n] = np.arange(7)[b:b + n]
        m.refs[m.table[b, :n]] = 1
    eng.block_table.copy_(i32(m.table)), eng.page_refs.copy_(i32(m.refs))
    same(eng, m)
    eng.fork(i32([0, 0, 0, 0, 0])), m.fork(np.asarray([0, 0, 0, 0, 0]))      # two pages for four copies: the first two get them
    same(eng, m)
    assert (eng.block_table[3] == -1).all() and eng.seq_len[3].item() == 20
    eng.reserve(40), m.reserve(40)
    same(eng, m)
    eng.close()


def test_entries_that_nobody_counted():
    """A page without references in a table: an error bit, and no count below zero."""
    eng = pooled(20, 2, 4)
    load(eng, [30, 30])
    eng.block_table[0, :3] = i32([5, 5, 6])
    eng.page_refs[5] = 1
    m = Model(eng)
    eng.free_pages(i32([0, 0]), i32([END, END])), m.free([0, 0], [END, END])
    same(eng, m)
    assert (eng.page_refs == 0).all()
    eng.close()


def test_rows_behind_the_batch():
    """Tables of sequences that are not in the batch are renamed by a compaction and left alone by all other calls."""
    eng = pooled(40, 6, 5)
    load(eng, [30, 40, 50, 60, 70, 20])
    eng.reserve(10)
    load(eng, [33, 44, 55])
    m = Model(eng)
    for b in range(6):
        m.table[b, :5] = np.arange(5) * 7 + b
    m.refs[:] = np.bincount(m.table.reshape(-1), minlength=40)
    eng.block_table.copy_(i32(m.table)), eng.page_refs.copy_(i32(m.refs))
    parent = np.asarray([1, 1, 1, 0, 0, 0])
    eng.fork(i32(parent)), m.fork(parent)
    same(eng, m)
    eng.free_pages(i32([16] * 6), i32([END] * 6)), m.free([16] * 6, [END] * 6)
    same(eng, m)
    eng.reserve(3), m.reserve(3)
    same(eng, m)
    live, to = m.compact()
    assert eng.compact().item() == live
    same(eng, m)
    eng.close()


def test_the_callers_own_holds():
    """A page that the caller counts for itself is not taken, and is found again by its new number."""
    eng = pooled(30, 2, 4)
    load(eng, [20, 40])
    eng.page_refs[[0, 17, 29]] = 1
    m = Model(eng)
    eng.reserve(20), m.reserve(20)
    same(eng, m)
    moved = torch.zeros(30, dtype=torch.int32, device="cuda:0")
    eng.compact(moved)
    live, to = m.compact()
    same(eng, m)
    assert (moved.cpu().numpy() == to).all() and to[29] >= 0 and to[29] < live
    eng.close()


@pytest.mark.parametrize("pages", [1, 63, 64, 65, 4095, 4096, 4097, 9000])
def test_pool_sizes(pages):
    eng = pooled(pages, 6, 40, seed=pages)
    rng = np.random.default_rng(pages)
    load(eng, [int(x) for x in rng.integers(1, 600, 6)])
    m = Model(eng)
    held = rng.random(pages) < 0.7      # (somebody's)
    eng.page_refs.copy_(i32(held))
    m.refs[:] = held
    for extra in (1, 500):
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


def test_a_large_pool():
    """More pages than 64 times 4096, of which the free ones lie far apart and behind the first 262144."""
    pages = 270001
    eng = pooled(pages, 3, 700)
    load(eng, [1, 5000, 40])
    held = np.ones(pages, np.int32)
    held[[3, 70000, 70001, 200000]] = 0
    held[262140:262160] = 0
    held[269000:] = 0
    eng.page_refs.copy_(i32(held))
    free = [int(p) for p in np.nonzero(held == 0)[0]]
    eng.reserve(600)
    table = eng.block_table.cpu().numpy()
    want = np.full((3, 700), -1, np.int32)
    o = 0
    for b, L in enumerate((0, 4999, 39)):
        for i in range(L // 16, (L + 600 + 15) // 16):
            want[b, i] = free[o]
            o += 1
    assert (table == want).all()
    refs = held.copy()
    refs[free[:o]] = 1
    assert (eng.page_refs.cpu().numpy() == refs).all()
    eng.page_refs[torch.arange(0, pages, 3, device="cuda:0")] = 0
    eng.page_refs[eng.block_table[eng.block_table >= 0].long()] = 1
    refs = eng.page_refs.cpu().numpy().copy()
    before = eng.kc.view(pages, -1)[:, :8].cpu().numpy().copy()
    moved = torch.zeros(pages, dtype=torch.int32, device="cuda:0")
    live = eng.compact(moved).item()
    assert live == int((refs != 0).sum())
    to = np.where(refs != 0, np.arange(pages), -1)
    src, dst = np.nonzero(refs[live:])[0] + live, np.nonzero(refs[:live] == 0)[0]
    to[src] = dst
    assert (moved.cpu().numpy() == to).all()
    after = eng.kc.view(pages, -1)[:, :8].cpu().numpy()
    assert (after[to[to >= 0]] == before[to >= 0]).all()
    assert (eng.block_table.cpu().numpy() == np.where(table >= 0, to[np.maximum(table, 0)], -1)).all()
    eng.close()


def test_captured_and_replayed():
    """A turnover of pages recorded once and replayed on states that have changed."""
    eng = pooled(60, 5, 8, 2, 64, 2)
    load(eng, [70, 33, 20, 50, 10])
    eng.reserve(1)
    parent, first, end = i32([0, 0, 0, 3, 3]), i32([1000, 0, 0, 1000, 0]), i32([END] * 5)
    m = Model(eng)
    eng.free_pages(first, end), eng.fork(parent), eng.reserve(20)
    m.free(first.tolist(), end.tolist()), m.fork(parent.tolist()), m.reserve(20)
    same(eng, m)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        eng.free_pages(first, end)
        eng.fork(parent)
        eng.reserve(20)
        eng.compact()
    for lens, par in (([70, 1, 1, 50, 1], [0, 0, 0, 3, 3]), ([90, 2, 2, 17, 9], [3, 3, -1, 3, 3]), ([16, 100, 2, 17, 9], [0, 1, 1, 1, 0])):
        eng.seq_len.copy_(i32(lens)), parent.copy_(i32(par))
        m.state["seq_len"][:] = lens
        g.replay()
        m.free(first.tolist(), end.tolist()), m.fork(np.asarray(par)), m.reserve(20)
        live, to = m.compact()
        same(eng, m, lens)
        assert eng.live_pages.item() == live
    eng.close()


def test_refusals_from_python():
    eng = pooled(20, 4, 4)
    load(eng, [10, 10, 10])
    ok = i32([0, 1, 2])
    for bad in (ok[:2], ok.long(), ok.cpu(), ok.view(1, 3), i32([0, 1, 2, 0, 1, 2])[::2]):
        with pytest.raises(ValueError):
            eng.fork(bad)
        with pytest.raises(ValueError):
            eng.free_pages(ok, bad)
    for bad in (i32([0] * 19), torch.zeros(20, device="cuda:0"), torch.zeros(20, dtype=torch.int32)):
        with pytest.raises(ValueError):
            eng.compact(bad)
    with pytest.raises(Exception):
        eng.reserve(-1)
    eng.close()
