"""hs_attention_window and hs_set_window against the definition in 64 bits: windows and sinks of all relations to tiles,
pages and partitions, drafts, trees, chunks and single tokens, empty rows, values that nobody may see."""
import numpy as np
import pytest
import torch

from window_common import chain, check, engine, gathered, lay_out, lay_out_chunk, queries, random_tree, reference

pytestmark = pytest.mark.gpu

HEADS = [(4, 4, 64), (7, 1, 64), (28, 4, 128), (8, 1, 128), (3, 3, 128), (10, 2, 64)]


def run(eng, m, q, window, sinks, chunk=0, out=None):
    out = torch.full((eng.max_rows, q.shape[1]), 7.0, device="cuda:0", dtype=q.dtype) if out is None else out
    full = torch.zeros(eng.max_rows, q.shape[1], device="cuda:0", dtype=q.dtype)
    full[:m] = q
    eng.attention_window(0, full, out, window, sinks, chunk)
    torch.cuda.synchronize()
    assert (out[m:] == 7.0).all()           # rows behind the last one
    return out


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (2, 1), (16, 0), (31, 4), (32, 33), (33, 16), (64, 64), (100, 3), (257, 130),
                                          (4096, 0), (1 << 30, 1 << 30)])
def test_single_tokens(heads, window, sinks):
    lens = [1, 2, 15, 16, 17, 33, 64, 65, 129, 300, 700]
    eng = engine(*heads, lens, 1)
    pars = [chain(0)] * len(lens)
    m = lay_out(eng, lens, pars)
    q = queries(m, eng)
    check(run(eng, m, q, window, sinks), eng, lens, pars, q, window, sinks)
    eng.close()


@pytest.mark.parametrize("heads", [(28, 4, 128), (7, 1, 64), (4, 4, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 4), (2500, 0), (4000, 1100), (1 << 30, 0), (300, 1 << 30)])
def test_single_tokens_behind_long_texts(heads, window, sinks):
    """Several partitions per sequence, of few sequences."""
    lens = [1, 4999, 2048, 2049, 3500] * (8 // heads[1])
    eng = engine(*heads, lens, 1)
    pars = [chain(0)] * len(lens)
    m = lay_out(eng, lens, pars)
    q = queries(m, eng)
    eng.workspace.fill_(0xFF)
    check(run(eng, m, q, window, sinks), eng, lens, pars, q, window, sinks)
    eng.close()


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 0), (5, 2), (20, 4), (40, 600), (63, 1), (64, 1), (300, 4)])
def test_drafts_and_trees(heads, window, sinks):
    """Chains of 1 .. 31 tokens, trees of up to 25 nodes (some with windows shorter than the draft), a sequence without rows."""
    rng = np.random.default_rng(window)
    lens = [1, 40, 65, 97, 500, 333, 210, 1000]
    pars = [random_tree(9, rng), chain(0), chain(30), None, random_tree(25, rng), chain(8), random_tree(2, rng), chain(13)]
    eng = engine(*heads, lens, 32)
    m = lay_out(eng, lens, pars)
    q = queries(m, eng)
    check(run(eng, m, q, window, sinks), eng, lens, pars, q, window, sinks)
    eng.close()


@pytest.mark.parametrize("window", [7, 70])
def test_sixty_four_nodes(window):
    """The most nodes and query rows that a sequence may have."""
    rng = np.random.default_rng(2)
    lens, pars = [3, 130, 64], [random_tree(63, rng), random_tree(63, rng), chain(31)]
    eng = engine(8, 2, 64, lens, 63, c_max=2)
    m = lay_out(eng, lens, pars)
    q = queries(m, eng)
    check(run(eng, m, q, window, 4), eng, lens, pars, q, window, 4)
    eng.close()


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("window,sinks,chunk", [(1, 0, 40), (10, 4, 40), (33, 0, 17), (64, 70, 300), (500, 4, 300), (4096, 0, 111)])
def test_chunks(heads, window, sinks, chunk):
    """Up to `chunk` consecutive tokens per sequence, shorter ones and none among them; a launch shaped for fewer rows than
    there are computes all of them."""
    lens = [1, 2, 100, 333, 64, 17]
    counts = [chunk, 1, chunk // 2, chunk, 0, 7]
    eng = engine(*heads, lens, 1, max_rows=sum(counts) + 5, spare=chunk)
    pars = [np.arange(-1, n - 1) for n in counts]
    m = lay_out_chunk(eng, counts)
    q = queries(m, eng)
    got = run(eng, m, q, window, sinks, chunk)
    check(got, eng, lens, pars, q, window, sinks, chunk=True)
    assert torch.equal(run(eng, m, q, window, sinks, 1), got)
    eng.close()


@pytest.mark.parametrize("window,sinks", [(15900, 100), (15000, 1001)])
def test_long_walks(window, sinks):
    """One walk over as many keys as there are in a workgroup's list of pages, and one more than that in partitions."""
    lens = [16300, 40, 18000] + [33] * 253
    eng = engine(8, 1, 64, lens, 9)
    pars = [chain(8), chain(3), chain(0)] + [chain(1)] * 253
    m = lay_out(eng, lens, pars)
    q = queries(m, eng)
    check(run(eng, m, q, window, sinks), eng, lens, pars, q, window, sinks)
    eng.close()


def test_a_cache_of_more_than_four_gigabytes():
    """17 texts of 131072 tokens in shuffled pages: offsets beyond 32 bits, whole walks, wavefronts', partitions and a chunk."""
    n, nodes, batch = 131072, 5, 17
    lens = [n - 3 * i for i in range(batch)]
    eng = engine(8, 8, 128, lens, nodes)
    assert eng.kc.numel() * 2 > 1 << 32
    pars = [chain(nodes - 1)] * batch
    for window, sinks, chunk in ((100, 4, 0), (300, 5, 0), (5000, 40, 0), (300, 5, nodes)):
        m = lay_out_chunk(eng, [nodes] * batch) if chunk else lay_out(eng, lens, pars)
        q = queries(m, eng)
        check(run(eng, m, q, window, sinks, chunk), eng, lens, pars, q, window, sinks, chunk=bool(chunk))
    eng.close()


def test_large_scores():
    """Scores of a few hundred (one key has all the weight) and a long window over many partitions."""
    lens, pars = [3000, 2999], [chain(4), chain(0)]
    eng = engine(14, 2, 128, lens, 5)
    m = lay_out(eng, lens, pars)
    for scale in (0.0, 30.0):
        q = queries(m, eng, scale=scale)
        check(run(eng, m, q, 2500, 8), eng, lens, pars, q, 2500, 8)
    eng.close()


@pytest.mark.parametrize("heads,batch", [((8, 2, 64), 256), ((40, 8, 128), 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (20, 4), (64, 70), (300, 5), (8000, 8)])
def test_large_batches(heads, batch, window, sinks):
    """As many (sequence, KV head) pairs as a launch has places: a workgroup for each, which writes the result itself (up to 16000 keys in
    sinks and window); some sequences without rows, in drafts of one to 17 nodes."""
    rng = np.random.default_rng(window)
    nodes = 17
    lens = [int(x) for x in rng.integers(1, 700, batch)]
    pars = [None if i % 7 == 3 else chain(0) if i % 3 == 0 else random_tree(int(rng.integers(2, nodes + 1)), rng) for i in range(batch)]
    eng = engine(*heads, lens, nodes)
    m = lay_out(eng, lens, pars)
    q = queries(m, eng)
    eng.workspace.fill_(0xFF)
    out = run(eng, m, q, window, sinks)
    check(out, eng, lens, pars, q, window, sinks)
    # the output may be the queries, and a row's bits do not depend on its neighbours
    buf = torch.full((eng.max_rows, q.shape[1]), 7.0, device="cuda:0", dtype=q.dtype)
    buf[:m] = q
    eng.attention_window(0, buf, buf, window, sinks)
    assert torch.equal(buf, out)
    alone = [p if p is None else chain(0) for p in pars]
    starts = np.cumsum([0] + [0 if p is None else len(p) for p in pars])[:-1]
    first = [int(s) for s, p in zip(starts, pars) if p is not None]
    m = lay_out(eng, lens, alone)
    assert torch.equal(run(eng, m, q[first], window, sinks)[:m], out[first])
    eng.close()


@pytest.mark.parametrize("heads", [(7, 1, 64), (8, 1, 128)])
@pytest.mark.parametrize("rate", [0.1, 0.4, 1.0])
def test_scores_that_rise_or_fall_along_the_keys(heads, rate):
    """The running maximum moves all the time, a little or a lot per tile (one product per score, so that an exponent of 500 is off
    by 2^-24 of itself for each of two roundings: 6e-5)."""
    lens, nodes = [600, 350], 5
    for chunk in (0, nodes):
        eng = engine(*heads, lens, nodes, spare=nodes)
        hq, hkv, hd = heads
        k = eng.kc.view(torch.bfloat16).view(eng.n_layers, eng.n_blocks, hkv, 16, hd)[0]
        k.zero_()
        for b, n in enumerate(lens):
            pages = eng.block_table[b, :(n + nodes) // 16 + 1].long()
            at = torch.arange(len(pages) * 16, device="cuda:0", dtype=torch.float32).view(-1, 1, 16)
            k[pages, :, :, 0] = (at * rate).expand(-1, hkv, -1).to(torch.bfloat16)
        pars = [chain(nodes - 1), chain(nodes - 1)]
        m = lay_out_chunk(eng, [nodes, nodes]) if chunk else lay_out(eng, lens, pars)
        q = queries(m, eng)
        for window, sinks in ((4096, 0), (200, 4)):
            check(run(eng, m, q, window, sinks, chunk), eng, lens, pars, q, window, sinks, chunk=bool(chunk))
        eng.close()


def test_a_rows_result_does_not_depend_on_the_other_rows():
    """Chains decoded token by token and as one draft: the same bits (what makes greedy speculative decoding equal plain greedy
    decoding); with few and many partitions, with windows below and above the draft's length."""
    for heads in ((28, 4, 128), (4, 4, 64)):
        lens, k = [90, 1000, 517, 1], 12
        eng = engine(*heads, lens, k + 1)
        for window, sinks in ((5, 2), (100, 4), (700, 40)):
            m = lay_out(eng, lens, [chain(k)] * len(lens))
            q = queries(m, eng)
            whole = run(eng, m, q, window, sinks).clone().view(-1)[:m * q.shape[1]].view(len(lens), k + 1, -1)
            for i in range(k + 1):
                longer = [n + i for n in lens]
                eng.seq_len.copy_(torch.tensor(longer, dtype=torch.int32))
                m1 = lay_out(eng, longer, [chain(0)] * len(lens))
                one = run(eng, m1, q.view(len(lens), k + 1, -1)[:, i].contiguous(), window, sinks)
                assert torch.equal(one[:m1], whole[:, i]), (heads, window, i)
            eng.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        eng.close()


def test_chunks_cut_differently_give_the_same_bits():
    lens, n = [70, 200, 1], 150
    eng = engine(12, 2, 128, lens, 1, max_rows=3 * n, spare=n)
    for window, sinks in ((9, 0), (130, 5)):
        m = lay_out_chunk(eng, [n] * 3)
        q = queries(m, eng)
        whole = run(eng, m, q, window, sinks, n).clone().view(3, n, -1)
        at = 0
        for step in (1, 31, 64, 54):
            eng.seq_len.copy_(torch.tensor([x + at for x in lens], dtype=torch.int32))
            mm = lay_out_chunk(eng, [step] * 3)
            part = run(eng, mm, q.view(3, n, -1)[:, at:at + step].reshape(mm, -1), window, sinks, step)
            assert torch.equal(part[:mm].view(3, step, -1), whole[:, at:at + step]), (window, step)
            at += step
        eng.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
    eng.close()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see_has_no_influence(bad):
    """NaN and infinities in K and V of slots that a row does not see: behind its window (inside the same page and tile), behind the
    last row, and in draft nodes that are no ancestors of it."""
    lens = [100, 300, 20]
    tree = np.asarray([-1, 0, 0, 1, 2, 3])               # two branches: nodes 1 3 5 and 2 4
    pars = [tree, chain(3), tree]
    window, sinks = 37, 3
    eng = engine(7, 1, 128, lens, 6, spare=8)
    m = lay_out(eng, lens, pars)
    q = queries(m, eng)
    clean = check(run(eng, m, q, window, sinks), eng, lens, pars, q, window, sinks)
    kc = eng.kc.view(torch.bfloat16).view(eng.n_blocks, 1, 16, 128)
    vc = eng.vc.view(torch.bfloat16).view(eng.n_blocks, 1, 128, 16)

    def spoil(b, slot):
        page = int(eng.block_table[b, slot // 16])
        kc[page, :, slot % 16] = bad
        vc[page, :, :, slot % 16] = bad

    for b, n in enumerate(lens):
        for slot in range(sinks, n - window):              # behind the window of every row
            spoil(b, slot)
        for slot in range(n - 1 + len(pars[b]), 16 * ((n - 1 + len(pars[b]) + 15) // 16)):
            spoil(b, slot)
    got = run(eng, m, q, window, sinks)[:m].double()
    assert torch.isfinite(got).all()
    check(got, eng, lens, pars, q, window, sinks, blocked=lambda b: torch.zeros(400, dtype=torch.bool).numpy())
    # a node's own values: only rows that see it may change
    spoil(0, 99 + 2)
    got = run(eng, m, q, window, sinks)[:m].double()
    for row, sees in ((0, False), (1, False), (2, True), (3, False), (4, True), (5, False)):
        if sees:
            assert not torch.isfinite(got[row]).all()
        else:
            assert (got[row] - clean[row]).abs().max() < 0.05 and torch.isfinite(got[row]).all()
    assert torch.isfinite(got[6:]).all()
    eng.close()


def test_a_chunks_later_tokens_have_no_influence():
    lens, n = [50], 64
    eng = engine(7, 1, 128, lens, 1, max_rows=n, spare=n)
    m = lay_out_chunk(eng, [n])
    q = queries(m, eng)
    clean = run(eng, m, q, 20, 2, n)[:m].double()
    vc = eng.vc.view(torch.bfloat16).view(eng.n_blocks, 1, 128, 16)
    for slot in range(49 + 40, 49 + n):
        vc[int(eng.block_table[0, slot // 16]), :, :, slot % 16] = float("nan")
    got = run(eng, m, q, 20, 2, n)[:m].double()
    assert torch.isnan(got[40:]).all() and (got[:40] - clean[:40]).abs().max() < 0.05
    eng.close()


def test_rows_that_see_nothing_are_zero():
    """An empty ancestor mask with a window that holds no cached token, and pages that the table does not have."""
    lens, pars = [64, 200], [chain(2), chain(2)]
    eng = engine(7, 1, 128, lens, 3)
    m = lay_out(eng, lens, pars)
    q = queries(m, eng)
    eng.st["anc_mask"][1] = 0                                # node 1 of sequence 0
    out = run(eng, m, q, 1, 0)
    want = reference(eng, lens, pars, q, 1, 0)[0]
    assert (out[1] == 0).all()
    keep = [0, 2, 3, 4, 5]
    assert (out[keep].double() - want[keep]).abs().max() < 0.05
    # sequence 1 loses its last pages: its rows see what is left of their windows, or nothing
    m = lay_out(eng, lens, pars)
    eng.block_table[1, 11:] = -1                             # positions from 176 on
    eng.block_table[0, 2] = eng.n_blocks                     # positions 32 .. 47 of sequence 0
    lost = lambda b: np.arange(400) >= 176 if b else (np.arange(400) >= 32) & (np.arange(400) < 48)
    for window, sinks in ((10, 0), (40, 0), (10, 4), (500, 0)):
        out = run(eng, m, q, window, sinks)
        check(out, eng, lens, pars, q, window, sinks, blocked=lost)
        if (window, sinks) == (10, 0):
            assert (out[3:6] == 0).all()
    eng.close()


@pytest.mark.parametrize("heads", [(4, 1, 64), (8, 1, 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (1, 70), (3, 0), (3, 2)])
def test_a_sequence_that_has_outgrown_its_table(heads, window, sinks):
    """Positions beyond the table are not seen: of a window that lies there nothing is left, whatever the workspace held."""
    nodes = 5                                                # 20 or 40 query rows per KV head
    eng = engine(*heads, [74, 60], nodes)
    cap = eng.block_table.shape[1] * 16
    assert cap == 96
    table = eng.block_table[:, :6].clone()
    for chunk in (0, nodes):
        lens = [cap + 1, 61]                                 # sequence 0's rows lie at positions 96 .. 100
        eng.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        pars = [chain(nodes - 1), chain(nodes - 1)]
        m = lay_out_chunk(eng, [nodes, nodes]) if chunk else lay_out(eng, lens, pars)
        q = queries(m, eng)
        eng.workspace.fill_(0xFF)                            # (NaNs)
        out = run(eng, m, q, window, sinks, chunk)
        # the reference's sequence 0 has a longer table, of which nothing more is seen
        wide = eng.block_table
        eng.block_table = torch.cat([table, table[:, :1]], 1)
        check(out, eng, lens, pars, q, window, sinks, chunk=bool(chunk), blocked=lambda b: np.arange(200) >= (cap if b == 0 else 200))
        eng.block_table = wide
        if sinks == 0:
            assert (out[4].float() == 0).all()               # position 100: sees neither 94 nor 95
    eng.close()


def test_pages_behind_the_window_are_not_used():
    """Their table entries may be gone, or name a page that another sequence has."""
    lens, pars = [400, 410], [chain(3), chain(0)]
    for chunk in (0, 4):
        eng = engine(28, 4, 128, lens, 4, spare=4)
        m = lay_out(eng, lens, pars) if not chunk else lay_out_chunk(eng, [4, 1])
        q = queries(m, eng)
        before = run(eng, m, q, 100, 4, chunk).clone()
        first = 399 + 1 - 100                                # first position in the window of sequence 0's first row
        eng.block_table[0, 1:first // 16] = -1
        eng.block_table[1, 1:5] = int(eng.block_table[0, 24])
        assert torch.equal(run(eng, m, q, 100, 4, chunk), before)
        eng.close()


def test_fp32_activations():
    """The plain kernel with float queries, cache and output: as exact as fp32 is."""
    rng = np.random.default_rng(9)
    lens, pars = [1, 70, 200], [chain(0), random_tree(9, rng), chain(5)]
    eng = engine(8, 2, 64, lens, 9, precise=True)
    m = lay_out(eng, lens, pars)
    q = queries(m, eng)
    for window, sinks in ((1, 0), (4, 2), (50, 4), (1000, 0)):
        want, mag = reference(eng, lens, pars, q, window, sinks)
        got = run(eng, m, q, window, sinks)[:m].double()
        # products, exponentials and sums in 64 bits: the inputs' and the result's rounding, and 1e-6 for the scale in 32
        assert ((got - want).abs() <= 2.0 ** -24 * want.abs() + 2e-6 * mag + 1e-12).all(), (window, sinks)
    eng.block_table[2, 3:9] = -1                             # positions 48 .. 143 of sequence 2
    lost = lambda b: (np.arange(400) >= 48) & (np.arange(400) < 144) & (b == 2)
    for window, sinks in ((30, 60), (180, 0)):
        want, mag = reference(eng, lens, pars, q, window, sinks, blocked=lost)
        got = run(eng, m, q, window, sinks)[:m].double()
        assert ((got - want).abs() <= 2.0 ** -24 * want.abs() + 2e-6 * mag + 1e-12).all(), (window, sinks)
    eng.close()


def test_streams_and_graphs():
    """On a stream of its own, and recorded: every replay gives the eager result for the inputs it finds."""
    lens, pars = [300, 77], [chain(5), chain(0)]
    eng = engine(12, 2, 128, lens, 6)
    m = lay_out(eng, lens, pars)
    qs = [queries(eng.max_rows, eng, seed=s) for s in range(4)]
    eager = [run(eng, m, q[:m], 50, 4).clone() for q in qs]
    q, out = qs[0].clone(), torch.full_like(eager[0], 7.0)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        eng.attention_window(0, q, out, 50, 4)
    side.synchronize()
    assert torch.equal(out[:m], eager[0][:m])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        eng.attention_window(0, q, out, 50, 4)
    for i in (1, 2, 3, 1):
        q.copy_(qs[i])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:m], eager[i][:m]), i
        eng.attention_window(0, qs[0], torch.zeros_like(out), 20, 0)          # the program's own call in between
    eng.close()


def test_the_output_may_be_the_queries():
    lens, pars = [300, 77], [chain(5), chain(0)]
    for chunk in (0, 6):
        eng = engine(12, 2, 128, lens, 6, spare=6)
        m = lay_out(eng, lens, pars) if not chunk else lay_out_chunk(eng, [6, 1])
        q = queries(m, eng)
        want = run(eng, m, q, 50, 4, chunk)[:m]
        full = torch.zeros(eng.max_rows, q.shape[1], device="cuda:0", dtype=q.dtype)
        full[:m] = q
        eng.attention_window(0, full, full, 50, 4, chunk)
        assert torch.equal(full[:m], want)
        eng.close()


def test_binding_refuses_tensors():
    eng = engine(4, 4, 64, [20], 1)
    q = torch.zeros(1, 256, device="cuda:0", dtype=torch.bfloat16)
    for a, b in ((q.float(), q), (q, q.float()), (q.float(), q.float()), (torch.zeros(1, 512, device="cuda:0", dtype=torch.bfloat16)[:, ::2], q)):
        with pytest.raises(ValueError):
            eng.attention_window(0, a, b, 4)
    with pytest.raises(ValueError):
        eng.set_window([4, 4])
    for a, b in ((q.cpu(), q), (q, q.cpu())):                # memory that the device does not have
        with pytest.raises(ValueError, match="cuda"):
            eng.attention_window(0, a, b, 4)
    eng.close()


# ---------------------------------------------------------------- the model's path

def _toy(**kw):
    from hs_inputs import CONFIG_SHAPES, config_seed, make_weights, rope_table
    from paper_2508_18588_amd.runtime import Engine
    shape = CONFIG_SHAPES[1]
    return shape, Engine(shape, make_weights(shape, config_seed(1)), rope_table(1024, shape.head_dim), **kw)


def _decode(eng, prompts, hists, pol, budget, window, sinks):
    eng.set_window(window, sinks)
    eng.load_sequences(prompts, [budget] * len(prompts))
    eng.set_history(hists)
    eng.prefill(prompts)
    steps = 0
    while int(eng.budget_left[:len(prompts)].max()) > 0:
        eng.step(pol)
        steps += 1
        assert steps <= 2 * budget
    torch.cuda.synchronize()
    assert eng.poll_error() == 0
    return [eng.tokens[b, :len(p) + budget].cpu().numpy() for b, p in enumerate(prompts)], steps


@pytest.mark.parametrize("window,sinks", [(24, 4), ([16, 0], 2)])
def test_greedy_speculative_decoding_equals_plain_decoding_with_windows(window, sinks):
    from hs_inputs import history_with_context, make_prompts, mutate
    from paper_2508_18588_amd.runtime import Policy
    shape, eng = _toy(max_batch=3, k_max=8, c_max=1, max_len=200, shuffle_pages_seed=5)
    prompts = [p for p in make_prompts(3, 60, shape.vocab, seed=6)]
    none = [[np.zeros(0, np.int32)] for _ in prompts]
    plain, n_plain = _decode(eng, prompts, none, Policy(window=8, k_fixed=0, k_max=8), 60, window, sinks)
    rng = np.random.default_rng(4)
    hists = [[history_with_context(p, mutate(t[len(p):], 0.1, 0.0, shape.vocab, rng), 8)] for p, t in zip(prompts, plain)]
    spec, n_spec = _decode(eng, prompts, hists, Policy(window=8, m_min=3, k_fixed=8, k_max=8), 60, window, sinks)
    for a, b in zip(plain, spec):
        assert (a == b).all()
    assert n_spec < n_plain
    full, _ = _decode(eng, prompts, none, Policy(window=8, k_fixed=0, k_max=8), 60, None, 0)
    assert any((a != b).any() for a, b in zip(plain, full))       # (the window changes what the model says)
    eng.close()


def test_a_recorded_step_with_windows():
    """Decode steps replayed from a graph that was recorded with windows emit what eager steps emit; a window that is set
    afterwards does not change the graph."""
    from hs_inputs import make_prompts
    from paper_2508_18588_amd.runtime import Policy
    shape, eng = _toy(max_batch=3, k_max=4, c_max=1, max_len=200, shuffle_pages_seed=5)
    prompts, pol = [p for p in make_prompts(3, 60, shape.vocab, seed=6)], Policy(window=8, k_fixed=4, k_max=4)
    hists = [[np.concatenate([p[-7:], np.arange(100, 140, dtype=np.int32)])] for p in prompts]
    want, steps = _decode(eng, prompts, hists, pol, 30, 24, 4)

    def load():
        eng.load_sequences(prompts, [30] * 3)
        eng.set_history(hists)
        eng.prefill(prompts)

    load()
    eng.set_rows_hint(15)
    eng.step(pol)
    graph = eng.capture_step(pol)
    load()
    eng.set_window(None)
    for _ in range(steps):
        graph.replay()
        eng.poll_error()                                     # (the program synchronises in between)
    torch.cuda.synchronize()
    for b, t in enumerate(want):
        assert (eng.tokens[b, :len(t)].cpu().numpy() == t).all()
    eng.close()


def test_verify_with_windows_against_the_fp32_mode():
    """Logits of a step of trees: MFMA kernels against plain kernels, whose window attention is checked on its own above."""
    from gpu_common import derived_logit_tol
    rng = np.random.default_rng(3)
    got = []
    for precise in (False, True):
        shape, eng = _toy(max_batch=4, k_max=8, c_max=2, max_len=300, shuffle_pages_seed=5, precise=precise)
        eng.set_window([20, 50], 3)
        toks = [np.random.default_rng(b).integers(0, shape.vocab, n).astype(np.int32) for b, n in enumerate((40, 150, 260, 1))]
        eng.load_sequences(toks, [50] * 4)
        eng.prefill(toks)
        rng = np.random.default_rng(3)
        pars = [random_tree(17, rng) for _ in toks]
        from window_common import depths
        m = eng.set_rows([dict(tok=np.concatenate([t[-1:], rng.integers(0, shape.vocab, 16).astype(np.int32)]), parent=p,
                               pos=len(t) - 1 + depths(p)) for t, p in zip(toks, pars)])
        eng.verify()
        torch.cuda.synchronize()
        got.append(eng.logits[:m].double().cpu())
        eng.close()
    assert (got[0] - got[1]).abs().max() < derived_logit_tol(shape, 2)


def test_prefill_with_windows():
    """The cache after hs_prefill: within the logits' tolerance of the one that chains through hs_verify leave, and the same bits
    however the text is cut."""
    from gpu_common import LOGIT_TOL
    shape, eng = _toy(max_batch=3, k_max=8, c_max=1, max_len=320, shuffle_pages_seed=5, max_rows=400)
    toks = [np.random.default_rng(b).integers(0, shape.vocab, n).astype(np.int32) for b, n in enumerate((300, 37, 129))]
    eng.set_window([30, 64], 4)
    caches = []
    for chunk in (0, 128, 50, 7):
        eng.kc.zero_()
        eng.vc.zero_()
        eng.load_sequences(toks, [8] * 3)
        if chunk:
            eng.prefill_chunked(chunk)
        else:
            eng.prefill(toks)
        torch.cuda.synchronize()
        kv = []
        for layer in range(2):
            for b, t in enumerate(toks):
                kv += [x.clone() for x in gathered(eng, b, len(t) - 1, layer)]
        caches.append(kv)
    for a, b in zip(caches[0], caches[1]):
        assert ((a - b).abs() <= LOGIT_TOL + 2e-2 * a.abs()).all()
    for other in caches[2:]:
        for a, b in zip(caches[1], other):
            assert torch.equal(a, b)
    eng.close()
