"""Shared prefixes at their borders: very long runs, prefixes that a member has not cached whole, and texts that replace those the prefixes were for."""
import numpy as np
import pytest
import torch

from test_gpu_group_rollout import GROUPS, MEMBERS, N, engine, model, start_forked  # noqa: F401  (the fixture)
from test_gpu_shared import ALL, attend, build
from window_common import chain, check, lay_out

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("holes", [False, True])
def test_runs_of_more_tiles_than_are_looked_up_at_a_time(hd, holes):
    """35000 keys in two runs of 547 tiles; with pages that there are none of in the first 512 of a run and behind them."""
    import paper_2508_18588_amd as hs
    eng, lens, pars, q = build((2, 1, hd), [0, 3], [35000], [5, 40, 17], [1, 2, -5], seed=hd)
    blocked = None
    if holes:
        gone = [3, 1021, 1023, 1024, 1025, 1093, 1094, 2117, 2118, 2186]
        for b in range(3):
            eng.block_table[b, gone] = -1
        at = np.zeros(36000, bool)
        for p in gone:
            at[16 * p:16 * p + 16] = True
        blocked = lambda b: at
    pre = hs.hs_shared_prefix(1, 3, 256, eng.shared.group_off, eng.shared.prefix_len)
    out = torch.zeros_like(q)
    hs.hs_attention_shared(eng.ctx, eng.c_cache, eng.c_seq, eng.c_step, hs.hs_shared_args(0, pre, q.data_ptr(), out.data_ptr()), eng.stream())
    check(out, eng, lens, pars, q, ALL, 0, blocked=blocked)
    check(attend(eng, q), eng, lens, pars, q, ALL, 0, blocked=blocked)
    eng.close()


def _rows(eng, lens, q, who):
    """The results of the members in `who`, a row each, when only these have rows."""
    lay_out(eng, lens, [chain(0) if b in who else None for b in range(len(lens))])
    return attend(eng, q[list(who)].contiguous())


def test_what_a_row_depends_on():
    """A prefix that all members have cached: a row's bits are its own, whoever else has rows.  One that a member has not cached whole is cut to
    what the members with rows have: the bits are those with a prefix of that length."""
    lens = [352 + 10, 352 + 33, 352 + 1, 352 + 60]
    eng, lens, pars, q = build((28, 4, 128), [0, 4], [352], [10, 33, 1, 60], [1] * 4, seed=21)
    assert lens[2] - 1 == 352
    full = attend(eng, q)
    for who in ([0], [0, 1], [1, 3], [0, 2, 3]):
        assert torch.equal(_rows(eng, lens, q, who), full[who])
    # member 2 has just been forked: its newest token is the prefix's last one
    lens[2] = 352
    eng.seq_len[2] = 352
    with_it, without = _rows(eng, lens, q, [0, 1, 2, 3]), _rows(eng, lens, q, [0, 1, 3])
    assert torch.equal(without, full[[0, 1, 3]])
    lens_dev = eng._shared_arrays[1]
    lens_dev[0] = 351      # (the hints stay: 320 keys in whole tiles, which all have)
    assert torch.equal(_rows(eng, lens, q, [0, 1, 2, 3]), with_it)
    for who in ([0], [0, 1], [1, 2], [0, 2, 3]):
        assert torch.equal(_rows(eng, lens, q, who), with_it[who])
    lens_dev[0] = 352
    check(_rows(eng, lens, q, [0, 1, 2, 3]), eng, lens, pars, q, ALL, 0)
    eng.close()


@pytest.mark.parametrize("recorded", [False, True])
def test_new_texts_share_nothing(model, recorded):  # noqa: F811
    """load_sequences() ends the sharing of the texts that it replaces, in recorded graphs, too: the next texts' tables are their own."""
    shape, w, rope, prompts = model
    B = GROUPS * MEMBERS
    eng = engine(model, pages=160)
    start_forked(eng, prompts)
    eng.reserve(5)
    rows = lambda lens: eng.set_rows([dict(tok=np.asarray([7 + b]), parent=np.asarray([-1]), pos=np.asarray([n - 1])) for b, n in enumerate(lens)])
    rows([len(p) for p in prompts for _ in range(MEMBERS)])
    eng.verify()
    torch.cuda.synchronize()
    if recorded:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            eng.verify()
    end = torch.full((B,), 2 ** 31 - 1, dtype=torch.int32, device="cuda:0")
    eng.free_pages(torch.zeros_like(end), end)
    rng = np.random.default_rng(2)
    texts = [rng.integers(0, shape.vocab, n).astype(np.int32) for n in (100, 120, 99, 130, 97, 111)]
    eng.load_sequences(texts, [N] * B)
    assert eng.shared is None
    eng.reserve(1, first=torch.zeros_like(end))
    eng.prefill_chunked(64)
    m = rows([len(t) for t in texts])
    g.replay() if recorded else eng.verify()
    torch.cuda.synchronize()
    got = eng.logits[:m].clone()
    assert eng.poll_error() == 0
    eng.set_shared_prefix(None)
    eng.verify()
    assert (got - eng.logits[:m]).abs().max() < 2e-2      # (the tolerance of the path)
    with pytest.raises(ValueError, match="no shared prefixes"):
        eng.attention_shared(0, torch.zeros(m, shape.n_q_heads * shape.head_dim, device="cuda:0", dtype=torch.bfloat16),
                             torch.zeros(m, shape.n_q_heads * shape.head_dim, device="cuda:0", dtype=torch.bfloat16))
    eng.close()


@pytest.mark.parametrize("own", [5900, 6000, 6100, 9000])
def test_few_long_texts_in_a_large_batch(own):
    """128 places of which four are taken: own keys in one walk or in partitions, as the table's length says; a row's bits are the same with all taken."""
    rng = np.random.default_rng(own)
    group = [own, 3000, 17, own // 2]
    lens_own = group + [int(x) for x in rng.integers(1, 40, 124)]
    kinds = [1, 3, -4, 2] + [1] * 124
    eng, lens, pars, q = build((4, 2, 64), [0, 4, 128], [300, 96], lens_own, kinds, seed=own, spare=0)
    full = attend(eng, q)
    check(full, eng, lens, pars, q, ALL, 0)
    few = pars[:4] + [None] * 124
    m = lay_out(eng, lens, few)
    out = attend(eng, q[:m].contiguous())
    assert torch.equal(out, full[:m])
    eng.close()
