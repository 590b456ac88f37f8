"""Paths of the window attention and of the probabilities that take certain sizes: infinities and NaNs where a draft's keys come in partitions
or whole for a large batch and in the plain kernel, chunks whose keys come in several runs, fewer long rows of logits than compute units, the
largest vocabularies, and more sequences than the device has places for."""
import numpy as np
import pytest
import torch

from paper_2508_18588_amd import HS_FLAG_REFERENCE_KERNELS, hs_set_flags
from test_gpu_probs import check as check_accept, distributions, drafted, uniforms
from window_common import bound, chain, engine, lay_out, lay_out_chunk, queries, random_tree, reference, visible

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def attend(eng, m, q, window, sinks, chunk=0):
    out = torch.full((eng.max_rows, q.shape[1]), 7.0, device="cuda:0", dtype=q.dtype)
    full = torch.zeros(eng.max_rows, q.shape[1], device="cuda:0", dtype=q.dtype)
    full[:m] = q
    eng.workspace.fill_(0xFF)
    eng.attention_window(0, full, out, window, sinks, chunk)
    torch.cuda.synchronize()
    assert (out[m:] == 7.0).all()
    return out[:m].double()


def caches(eng):
    """K [pages, hkv, 16, hd] and V [pages, hkv, hd, 16]."""
    sh = eng.shape
    return (eng.kc.view(torch.bfloat16).view(eng.n_blocks, sh.n_kv_heads, 16, sh.head_dim),
            eng.vc.view(torch.bfloat16).view(eng.n_blocks, sh.n_kv_heads, sh.head_dim, 16))


def expect(eng, lens, pars, q, window, sinks, spoiled, chunk=False):
    """Replaces some keys and values, and gives what the definition then says: (result without the replaced ones, bound, rows x elements that
    NaNs, +inf and -inf go into).  spoiled: (sequence, slot, KV head, dim, value) of V, with dim None for all of K at that place (value NaN)."""
    sh = eng.shape
    kc, vc = caches(eng)
    G, hd = sh.n_q_heads // sh.n_kv_heads, sh.head_dim
    out, mag = reference(eng, lens, pars, q, window, sinks, chunk=chunk)
    kind = torch.zeros(3, out.shape[0], sh.n_kv_heads, G, hd, dtype=torch.bool, device="cuda:0")
    starts = np.cumsum([0] + [0 if p is None else len(p) for p in pars])
    for b in {x[0] for x in spoiled}:
        vis = visible(int(lens[b]), pars[b], window, sinks, chunk)
        for s, slot, j, dim, value in spoiled:
            if s != b or slot >= vis.shape[1]:
                continue
            rows = torch.as_tensor(starts[b] + np.nonzero(vis[:, slot])[0], device="cuda:0")
            at = slice(None) if dim is None else dim
            kind[0 if value != value else 1 if value > 0 else 2, rows, j, :, at] = True
    for b, slot, j, dim, value in spoiled:
        page, at = int(eng.block_table[b, slot // 16]), slot % 16
        if dim is None:
            kc[page, j, at] = value
        else:
            vc[page, j, dim, at] = value
    return out, bound(out, mag), kind.view(3, out.shape[0], -1)


def agree(got, out, tol, kind):
    nan = kind[0] | (kind[1] & kind[2])
    pos, neg = kind[1] & ~nan, kind[2] & ~nan
    assert torch.isnan(got[nan]).all(), "NaN"
    assert (got[pos] == INF).all() and (got[neg] == -INF).all(), "infinities"
    rest = ~(nan | pos | neg)
    assert torch.isfinite(got[rest]).all(), "what is seen of no infinity or NaN"
    assert ((got - out).abs()[rest] <= tol[rest]).all(), (got - out).abs()[rest].max()


def _case(eng, m, lens, pars, q, window, sinks, spoiled, chunk=0):
    out, tol, kind = expect(eng, lens, pars, q, window, sinks, spoiled, chunk=bool(chunk))
    return attend(eng, m, q, window, sinks, chunk), out, tol, kind


# heads, nodes of the longest draft, sequences: wavefronts' partitions (at most 32 rows per KV head), workgroups', whole walks
DRAFTS = [((7, 1, 128), 4, 3), ((8, 2, 64), 7, 3), ((7, 1, 128), 9, 3), ((16, 2, 64), 31, 3), ((8, 1, 64), 9, 256), ((8, 1, 128), 25, 256)]


@pytest.mark.parametrize("heads,nodes,batch", DRAFTS)
@pytest.mark.parametrize("window,sinks", [(1500, 70), (200, 0), (610, 5)])
def test_infinities_and_nans_in_long_texts(heads, nodes, batch, window, sinks):
    rng = np.random.default_rng(nodes)
    lens = [3001, 899, 700] + [40] * (batch - 3)
    pars = [chain(nodes - 1), random_tree(nodes, rng), chain(0)] + [chain(0)] * (batch - 3)
    eng = engine(*heads, lens, nodes, spare=16)
    m = lay_out(eng, lens, pars)
    q = queries(m, eng)
    hkv = heads[1]
    for value in (INF, -INF, NAN):
        spoiled = []
        for b in (0, 1, 2):
            L, first = lens[b] - 1, max(0, lens[b] - window)
            if first > sinks + 6:
                spoiled += [(b, first - 1, 0, 3, value), (b, first - 6, 0, None, NAN), (b, sinks, hkv - 1, 5, value)]      # no row sees these
            spoiled += [(b, first, 0, 9, value), (b, first + 1, hkv - 1, 11, -value)]      # the root's row and its children's
            spoiled += [(b, L + len(pars[b]), 0, 13, value), (b, L + len(pars[b]) + 1, 0, None, NAN)]      # behind the last node
            if sinks:
                spoiled += [(b, sinks - 1, 0, 17, value)]
            if len(pars[b]) > 3:
                spoiled += [(b, L + 2, 0, 21, value), (b, L + 2, hkv - 1, 22, -value)]
                spoiled += [(b, L + 3, hkv - 1, 22, value), (b, L + len(pars[b]) - 1, hkv - 1, 23, value)]
        # either side of every partition's edge, of any length
        for edge in range(64, lens[0] - 1, 64):
            if lens[0] - window + nodes < edge:
                spoiled += [(0, edge - 1, 0, 24 + edge // 64 % 16, value), (0, edge, 0, 40 + edge // 64 % 16, value)]
        kc, vc = eng.kc.clone(), eng.vc.clone()
        agree(*_case(eng, m, lens, pars, q, window, sinks, spoiled))
        # a node's key
        eng.kc.copy_(kc), eng.vc.copy_(vc)
        agree(*_case(eng, m, lens, pars, q, window, sinks, [(0, lens[0] - 1 + 2, 0, None, NAN), (1, lens[1] - 1 + 1, hkv - 1, None, NAN)]))
        eng.kc.copy_(kc), eng.vc.copy_(vc)
    eng.close()


@pytest.mark.parametrize("heads", [(4, 1, 128), (6, 2, 64)])
@pytest.mark.parametrize("window,sinks", [(20000, 0), (20000, 1001), (16200, 5), (1 << 30, 3)])
def test_chunks_with_more_keys_than_a_run_of_tiles(heads, window, sinks):
    """Texts of 40000 tokens: a workgroup's walk is two or three runs of 512 tiles of 32 keys; beside a short text."""
    lens, counts = [40000, 777], [150, 41]
    eng = engine(*heads, lens, 1, max_rows=sum(counts), spare=max(counts))
    pars = [np.arange(-1, n - 1) for n in counts]
    m = lay_out_chunk(eng, counts)
    q = queries(m, eng)
    agree(*_case(eng, m, lens, pars, q, window, sinks, [], chunk=150))
    L, first = lens[0] - 1, max(0, lens[0] - window)
    for value in (INF, NAN):
        spoiled = [(0, first + i, 0, 3 * i, value) for i in (0, 1, 4, 9)]                  # the first run: rows up to 0, 1, 4, 9 see them
        spoiled += [(0, L + i, heads[1] - 1, 40 + i // 40, -value) for i in (3, 40, 149)]      # the last one: rows from 3, 40, 149 on
        spoiled += [(0, L - 9000, 0, 50, value), (1, 700 + 5, 0, 51, value), (1, 776 + 41, 0, 52, value)]
        if first:
            spoiled += [(0, first - 1, 0, 53, value), (0, sinks, 0, 54, value)]
        kc, vc = eng.kc.clone(), eng.vc.clone()
        agree(*_case(eng, m, lens, pars, q, window, sinks, spoiled, chunk=150))
        eng.kc.copy_(kc), eng.vc.copy_(vc)
    eng.close()


@pytest.mark.parametrize("vocab,rows", [(1000003, 60), (1048576, 49), (4100000, 13)])
def test_fewer_long_rows_than_compute_units(vocab, rows):
    """Rows too long and too many to be read twice from the caches by launches of their own, but fewer than there are compute units."""
    assert rows * vocab * 4 > 192 << 20
    eng = engine(1, 1, 64, [8] * 4, 1, vocab=vocab)
    x = torch.randn(rows, vocab, device="cuda:0") * 3
    x[rows // 2, 1000:900000] = -INF
    out, few = torch.empty(rows, vocab, device="cuda:0"), torch.empty(2, vocab, device="cuda:0")
    eng.probs(x, out, 0.8)
    for r in [rows // 2, *range(0, rows, 5)]:
        y = x[r].double() / 0.8
        want = torch.softmax(y, -1)
        # a sum's roundings: 16 of a lane's tokens, 6 joining lanes, one per 64 units of 1024 tokens (at most 63), 6 again; exponents as long as
        # the logits are far apart, and a few more for each exponential, product and quotient
        tol = want * 2.0 ** -24 * (110 + 2 * (y.amax() - y).clamp(max=200))
        assert ((out[r].double() - want).abs() <= tol + 2.0 ** -125).all()
    eng.probs(x[3:5], few, 0.8)
    assert torch.equal(few, out[3:5])
    eng.close()


def test_a_vocabulary_beyond_25_million():
    """More slices of sums than 48 KB of LDS hold, where sums are the last launch's own: two rejected children behind one launch of sums."""
    vocab, m = 26000003, 4
    eng = engine(1, 1, 64, [8], m, vocab=vocab)
    x = torch.randn(m, vocab, device="cuda:0")
    p, q = torch.empty_like(x), torch.empty_like(x)
    eng.probs(x * 9, p, 1.1)
    eng.probs(x * 8 + torch.randn(m, vocab, device="cuda:0"), q, 1.0)
    y = x[0].double() * 9
    want = torch.softmax((x[0] * 9).double() / float(np.float32(1.1)), -1)
    # (as for fewer long rows, with 25391 units: 397 one after the other)
    tol = want * 2.0 ** -24 * (450 + 2 * ((y.amax() - y) / 1.1).clamp(max=200))
    assert ((p[0].double() - want).abs() <= tol + 2.0 ** -125).all()
    par = np.asarray([-1, 0, 0, 0])
    toks = [np.asarray([0] + [int(t) for t in q[0].topk(3).indices], np.int32)]
    for accept in (0.0, 1.0 - 2.0 ** -24):
        for sample in (0.0, 0.3, 0.9999, 1.0 - 2.0 ** -24):
            for d in (q, None):
                check_accept(eng, [par], toks, p, d, np.full(m, accept), np.full(1, sample))
    eng.close()


@pytest.mark.parametrize("drawn", [True, False])
def test_more_sequences_than_workgroups_that_sum(drawn):
    rng, vocab, n = np.random.default_rng(8), 300, 1500
    eng = engine(1, 1, 64, [8] * n, 4, vocab=vocab)
    pars = [None if b % 5 == 2 else chain(int(rng.integers(0, 4))) for b in range(n)]
    m = sum(len(x) for x in pars if x is not None)
    p, q = distributions(m, vocab, 3.0, 0.7, torch.float32, 9)
    toks = drafted(pars, q if drawn else p, vocab, rng)
    got = check_accept(eng, pars, toks, p, q if drawn else None, uniforms(rng, m), uniforms(rng, n))
    assert got["accept_len"].sum() > 0
    eng.close()


def test_the_plain_kernel_on_a_cache_of_16_bits():
    rng = np.random.default_rng(9)
    lens, pars = [1, 70, 300], [chain(0), random_tree(9, rng), chain(5)]
    eng = engine(8, 2, 64, lens, 9)
    m = lay_out(eng, lens, pars)
    q = queries(m, eng)
    hs_set_flags(eng.ctx, HS_FLAG_REFERENCE_KERNELS)
    eng._bind_workspace()
    for window, sinks in ((1, 0), (4, 2), (50, 4), (1000, 0)):
        agree(*_case(eng, m, lens, pars, q, window, sinks, []))
    L = lens[2] - 1
    agree(*_case(eng, m, lens, pars, q, 50, 4, [(2, L + 1 - 50, 0, 3, INF), (2, L - 50, 1, 4, NAN), (2, L + 2, 1, 5, NAN), (1, 69 + 9, 0, 6, NAN)]))
    eng.close()
