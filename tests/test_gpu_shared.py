"""Attention of sequences that share prefixes against its definition in 64 bits (window_common.bound: roundings of the weights, of partial
results and of the result), and what it must not depend on."""
import numpy as np
import pytest
import torch

from window_common import bound, chain, check, engine, lay_out, queries, random_tree, reference

pytestmark = pytest.mark.gpu
ALL = 1 << 30      # no window


def share(eng, off, pre):
    """Tables whose groups name the first sequence's pages for the first pre[g] positions, and the engine's prefixes."""
    for g, p in enumerate(pre):
        n = (p + 15) // 16
        for b in range(off[g] + 1, off[g + 1]):
            eng.block_table[b, :n] = eng.block_table[off[g], :n]
    eng.set_shared_prefix(off, pre)


def build(heads, off, pre, own, kinds, seed=0, spare=450, **kw):
    """An engine of groups off[] with prefixes pre[], own tokens own[b] and rows kinds[b] (a number of nodes, or parents).  spare: room in the tables for
    more tokens (with short tables every sequence reads the prefix for itself)."""
    hq, hkv, hd = heads
    group = np.full(len(own), -1)
    for g in range(len(pre)):
        group[off[g]:off[g + 1]] = g
    lens = [int(n) + (pre[g] if g >= 0 else 0) for n, g in zip(own, group)]
    rng = np.random.default_rng(seed)
    pars = [None if k is None else chain(k - 1) if isinstance(k, int) and k > 0 else random_tree(-k, rng) for k in kinds]
    nodes = max(1, max(len(p) for p in pars if p is not None))
    eng = engine(hq, hkv, hd, lens, nodes, seed=seed, spare=spare, **kw)
    share(eng, off, pre)
    m = lay_out(eng, lens, pars)
    return eng, lens, pars, queries(m, eng, seed=seed + 3)


def attend(eng, q, layer=0):
    out = torch.full_like(q, 7.0)
    eng.attention_shared(layer, q, out)
    torch.cuda.synchronize()
    assert eng.poll_error() == 0
    return out


CASES = [
    # heads, group bounds, prefixes, own tokens (the newest among them), nodes per sequence (negative: a random tree)
    ((4, 4, 64), [0, 4], [256], [1, 20, 33, 64], [1, 1, 1, 1]),
    ((4, 4, 64), [0, 1], [32], [1], [1]),                                   # a group of one sequence, a single run
    ((1, 1, 64), [0, 3], [31], [5, 40, 7], [1, 2, 3]),                      # a prefix below a tile
    ((12, 2, 128), [0, 7], [700], [900, 1900, 33, 1, 2, 500, 16], [1] * 7),
    ((28, 4, 128), [0, 3, 5], [100, 1000], [300, 1, 17, 64, 5], [1, 9, -17, 4, 1]),
    ((40, 8, 128), [0, 6], [517], [1, 15, 16, 17, 100, 31], [-17, -17, 1, -5, -9, -17]),
    ((8, 1, 128), [0, 5], [64], [1] * 5, [32, 31, 1, -30, 7]),              # eight heads per KV head, 256 rows of a sequence
    ((7, 1, 64), [0, 0, 4, 4, 6], [300, 96, 5, 33], [3, 4, 5, 6, 7, 8], [1, -3, 1, 2, 6, 1]),      # groups of none
    ((6, 3, 128), [2, 5], [200], [10, 20, 30, 40, 50, 60], [1, 2, 3, -4, 5, 1]),                   # sequences in no group
    ((4, 2, 64), [0, 4], [0], [30, 40, 50, 60], [1, 2, -3, 1]),             # nothing is shared
    ((5, 1, 128), [0, 33], [1111], list(range(1, 34)), [1] * 33),           # more members than lanes' halves, many row tiles
    ((28, 4, 128), [0, 70], [333], [1 + i % 9 for i in range(70)], [1 + i % 3 for i in range(70)]),      # more than 64 members
]


@pytest.mark.parametrize("spare", [0, 450])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_definition(case, spare):
    heads, off, pre, own, kinds = CASES[case]
    eng, lens, pars, q = build(heads, off, pre, own, kinds, seed=case, spare=spare)
    check(attend(eng, q), eng, lens, pars, q, ALL, 0)
    eng.close()


@pytest.mark.parametrize("spare", [0, 450])
@pytest.mark.parametrize("pre", [1, 15, 16, 17, 32, 33, 47, 48, 63, 64, 65, 255, 256, 257, 1023, 1025])
def test_prefixes_of_every_rest(pre, spare):
    eng, lens, pars, q = build((8, 2, 64), [0, 5], [pre], [1, 2, 16, 17, 40], [1, 3, -5, 1, 2], seed=pre, spare=spare)
    check(attend(eng, q), eng, lens, pars, q, ALL, 0)
    eng.close()


@pytest.mark.parametrize("hd", [64, 128])
def test_many_sequences_and_long_texts(hd):
    """A workgroup per (sequence, KV head), and partitions of long texts; prefixes in many runs and in one."""
    rng = np.random.default_rng(hd)
    own = [int(x) for x in rng.integers(1, 300, 128)]
    eng, lens, pars, q = build((16, 4, hd), list(range(0, 129, 16)), [int(x) for x in rng.integers(1, 2000, 8)], own, [1] * 128, seed=hd)
    check(attend(eng, q), eng, lens, pars, q, ALL, 0)
    eng.close()
    eng, lens, pars, q = build((8, 2, hd), [0, 2, 3], [2500, 40], [4000, 17, 9000], [1, -9, 4], seed=hd + 1)
    check(attend(eng, q), eng, lens, pars, q, ALL, 0)
    eng.close()
    own = [int(x) for x in rng.integers(1, 40, 96)]
    eng, lens, pars, q = build((16, 4, hd), [0, 64, 96], [1500, 700], own, [int(x) for x in rng.integers(1, 9, 96)], seed=hd + 2)
    check(attend(eng, q), eng, lens, pars, q, ALL, 0)
    eng.close()


def test_short_tables():
    """Tables of few pages: no room for a second partial result."""
    for cap in (1, 17, 60, 100, 130, 200):
        eng, lens, pars, q = build((4, 2, 64), [0, 3], [min(cap, 96)], [1 + cap // 3, 1, 2], [1, 1, 1], seed=cap, spare=0)
        check(attend(eng, q), eng, lens, pars, q, ALL, 0)
        eng.close()


@pytest.mark.parametrize("spare", [0, 450])
@pytest.mark.parametrize("gone", [[0], [0, 1], [2], [0, 3], [0, 1, 2, 3]])
def test_members_without_rows(gone, spare):
    """The first member that has rows is whose table is read: the others' entries may be gone."""
    kinds = [None if b in gone else [1, 3, -4, 2][b % 4] for b in range(6)]
    eng, lens, pars, q = build((4, 2, 128), [0, 4, 6], [300, 50], [20, 30, 40, 50, 60, 70], kinds, seed=9, spare=spare)
    for b in gone:
        eng.block_table[b] = -1
        eng.seq_len[b] = 0
    check(attend(eng, q), eng, lens, pars, q, ALL, 0)
    eng.close()


@pytest.mark.parametrize("spare", [0, 450])
def test_prefix_beyond_what_a_member_has_cached(spare):
    """It is cut to what all members with rows have cached: a prefix length that runs ahead does not change what a row sees."""
    eng, lens, pars, q = build((8, 2, 64), [0, 4], [320], [10, 20, 30, 40], [1, 2, -3, 1], seed=4, spare=spare)
    eng.set_shared_prefix([0, 4], [2 ** 31 - 1])
    for b in range(4):      # (all tables name the same pages for all positions that may be shared then)
        eng.block_table[b, :(min(lens) - 1) // 16] = eng.block_table[0, :(min(lens) - 1) // 16]
    check(attend(eng, q), eng, lens, pars, q, ALL, 0)
    eng.close()


@pytest.mark.parametrize("spare", [0, 450])
def test_missing_pages_are_not_seen(spare):
    eng, lens, pars, q = build((8, 2, 128), [0, 3, 4], [400, 64], [100, 200, 30, 90], [1, 9, -5, 2], seed=5, spare=spare)
    holes = {0: [2, 3, 9], 1: [2, 3, 9, 30], 2: [2, 3, 9], 3: [0, 5]}
    for b, pages in holes.items():
        for i, p in enumerate(pages):
            eng.block_table[b, p] = (-1, eng.n_blocks, 2 ** 30)[p % 3]
    eng.kc.view(torch.bfloat16)[:16] = float("nan")      # (whatever is read in their place counts for nothing)
    eng.vc.view(torch.bfloat16).view(eng.n_blocks, -1)[0] = float("nan")
    used = {int(p) for b in range(4) for p in eng.block_table[b, :(lens[b] + 20) // 16].tolist()}
    if 0 in used:      # page 0 is somebody's: it keeps finite numbers
        eng.kc.view(torch.bfloat16)[:16] = 0.5
        eng.vc.view(torch.bfloat16).view(eng.n_blocks, -1)[0] = 0.25

    def blocked(b):
        out = np.zeros(5000, bool)
        for p in holes[b]:
            out[16 * p:16 * p + 16] = True
        return torch.as_tensor(out)
    check(attend(eng, q), eng, lens, pars, q, ALL, 0, blocked=lambda b: blocked(b).numpy())
    eng.close()


@pytest.mark.parametrize("spare", [0, 450])
def test_nothing_to_see(spare):
    """Rows whose pages are all missing, sequences of no tokens: zeros."""
    eng, lens, pars, q = build((4, 2, 64), [0, 3], [64], [5, 6, 7], [1, 2, 1], seed=6, spare=spare)
    eng.block_table[:] = -1
    out = attend(eng, q)
    assert (out == 0).all()
    eng.seq_len[:] = 0
    assert (attend(eng, q) == 0).all()
    eng.close()


@pytest.mark.parametrize("spare", [40, 450])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_unseen_places_have_no_influence(bad, spare):
    """Slots behind the last node, draft nodes that are no ancestors, and other sequences' pages hold infinities or NaNs."""
    eng, lens, pars, q = build((8, 2, 128), [0, 3], [100], [9, 30, 44], [-6, 1, -9], seed=8, spare=spare)
    hkv, hd = 2, 128
    kc = eng.kc.view(torch.bfloat16).view(eng.n_blocks, hkv, 16, hd)
    vc = eng.vc.view(torch.bfloat16).view(eng.n_blocks, hkv, hd, 16)
    for b in range(3):
        total = lens[b] - 1 + len(pars[b])
        for t in range(total, 16 * ((total + 15) // 16) + 16):
            page = int(eng.block_table[b, t // 16])
            if page >= 0:
                kc[page, :, t % 16] = bad
                vc[page, :, :, t % 16] = bad
    check(attend(eng, q), eng, lens, pars, q, ALL, 0)
    eng.close()


@pytest.mark.parametrize("spare", [0, 450])
def test_seen_nonfinite_values_are_the_rows_own(spare):
    """A NaN in a prefix's values reaches every member's rows in that element, one in a sequence's own value its rows alone."""
    eng, lens, pars, q = build((4, 2, 64), [0, 3], [96], [20, 30, 40], [1, 2, 1], seed=3, spare=spare)
    vc = eng.vc.view(torch.bfloat16).view(eng.n_blocks, 2, 64, 16)
    vc[int(eng.block_table[1, (lens[1] - 5) // 16]), 1, 7, (lens[1] - 5) % 16] = float("nan")
    out = attend(eng, q).float().view(-1, 4, 64)
    want = torch.zeros_like(out, dtype=torch.bool)
    want[1:3, 2:, 7] = True      # sequence 1 has rows 1 and 2; KV head 1 serves heads 2 and 3
    assert (torch.isnan(out) == want).all()
    vc[int(eng.block_table[0, 2]), 0, 5, 3] = float("nan")
    out = attend(eng, q).float().view(-1, 4, 64)
    want[:, :2, 5] = True
    assert (torch.isnan(out) == want).all()
    eng.close()


def test_rows_do_not_depend_on_each_other():
    """A root's result has the same bits alone, next to draft nodes, and when other members have none; also with any row hint."""
    heads, off, pre, own = (28, 4, 128), [0, 4], [700], [100, 333, 5, 64]
    eng, lens, pars, q = build(heads, off, pre, own, [9, 9, 9, 9], seed=2)
    full = attend(eng, q).view(4, 9, -1)
    lay_out(eng, lens, [chain(0)] * 4)
    q0 = q.view(4, 9, -1)[:, 0].contiguous()
    assert torch.equal(attend(eng, q0), full[:, 0])
    lay_out(eng, lens, [None, chain(8), None, chain(2)])
    some = torch.cat([q.view(4, 9, -1)[1], q.view(4, 9, -1)[3, :3]]).contiguous()
    got = attend(eng, some)
    assert torch.equal(got[:9], full[1]) and torch.equal(got[9:], full[3, :3])
    lay_out(eng, lens, [chain(8)] * 4)
    for hint in (1, 7, 36, 100000):
        eng.set_rows_hint(hint)
        assert torch.equal(attend(eng, q).view(4, 9, -1), full)
    eng.close()


def test_small_hints_still_compute_everything():
    """Groups larger and prefixes longer than the hints say, straight through the C entry point."""
    import paper_2508_18588_amd as hs
    eng, lens, pars, q = build((28, 4, 128), [0, 40], [900], [1 + i % 5 for i in range(40)], [1 + i % 4 for i in range(40)], seed=12)
    for members, longest in ((1, 0), (1, 31), (2, 300), (40, 4000)):
        pre = hs.hs_shared_prefix(1, members, longest, eng.shared.group_off, eng.shared.prefix_len)
        out = torch.zeros_like(q)
        hs.hs_attention_shared(eng.ctx, eng.c_cache, eng.c_seq, eng.c_step, hs.hs_shared_args(0, pre, q.data_ptr(), out.data_ptr()), eng.stream())
        check(out, eng, lens, pars, q, ALL, 0)
    eng.close()


@pytest.mark.parametrize("spare", [0, 450])
def test_rows_behind_the_last_and_in_place(spare):
    eng, lens, pars, q = build((4, 2, 64), [0, 3], [64], [5, 6, 7], [1, 2, 1], seed=13, spare=spare, max_rows=40)
    want = attend(eng, q)
    big = torch.full((12, q.shape[1]), 3.0, device="cuda:0", dtype=torch.bfloat16)
    big[:4] = q
    eng.attention_shared(0, big, big)
    assert torch.equal(big[:4], want) and (big[4:] == 3.0).all()
    eng.close()


@pytest.mark.parametrize("spare", [0, 450])
def test_other_layers_and_streams(spare):
    eng, lens, pars, q = build((4, 2, 64), [0, 3], [100], [5, 60, 7], [1, 2, -4], seed=14, spare=spare, layers=3)
    for layer in range(3):
        check(attend(eng, q, layer), eng, lens, pars, q, ALL, 0, layer=layer)
    want, side = attend(eng, q, 1), torch.cuda.Stream()
    out = torch.zeros_like(q)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eng.attention_shared(1, q, out)
    side.synchronize()
    assert torch.equal(out, want)
    eng.close()


def test_precise_mode_reads_every_table():
    eng, lens, pars, q = build((4, 2, 64), [0, 3], [100], [5, 60, 7], [1, 2, -4], seed=15, precise=True)
    out, _ = reference(eng, lens, pars, q, ALL, 0)
    got = attend(eng, q).double()
    assert (got - out).abs().max() < 1e-5 * (1 + out.abs().max())      # (32-bit products, 64-bit sums)
    eng.close()


@pytest.mark.parametrize("spare", [0, 450])
def test_captured_and_replayed(spare):
    """A graph keeps the arrays, not their contents: prefixes and lengths may change between replays."""
    eng, lens, pars, q = build((8, 2, 64), [0, 3, 5], [200, 64], [50, 60, 70, 80, 90], [1, 2, 3, 1, 2], seed=16, spare=spare)
    out = torch.zeros_like(q)
    eng.attention_shared(0, q, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        eng.attention_shared(0, q, out)
    pre_dev = eng._shared_arrays[1]
    for pre in ([200, 64], [96, 0], [0, 32], [200, 64]):
        pre_dev[:2].copy_(torch.tensor(pre, dtype=torch.int32))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        check(out, eng, lens, pars, q, ALL, 0)
        again = torch.zeros_like(q)
        eng.attention_shared(0, q, again)
        assert torch.equal(again, out)
    eng.close()


@pytest.mark.parametrize("spare", [0, 450])
def test_a_graph_of_other_groups(spare):
    """Prefixes set anew leave the arrays that a recorded graph reads where they are; its groups that there are no more are empty."""
    eng, lens, pars, q = build((8, 2, 64), [0, 2, 4, 5], [200, 64, 96], [50, 60, 70, 80, 90], [1, 2, 3, 1, 2], seed=18, spare=spare)
    out = torch.zeros_like(q)
    eng.attention_shared(0, q, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        eng.attention_shared(0, q, out)
    for off, pre in (([0, 2], [160]), ([2, 4], [64]), ([0, 2, 4, 5], [200, 64, 96])):
        eng.set_shared_prefix(off, pre)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        check(out, eng, lens, pars, q, ALL, 0)
    eng.close()


@pytest.mark.parametrize("spare", [0, 450])
def test_text_beyond_the_table(spare):
    """Of a sequence that has outgrown its table a row sees what the table holds, in a prefix and in its own keys."""
    eng, lens, pars, q = build((8, 2, 64), [0, 3], [128], [30, 40, 50], [1, 1, 1], seed=19, spare=spare)
    cap = 16 * eng.max_blocks
    for ahead in (1, 17, 5000, 2 ** 31 - 2 - cap):
        eng.seq_len[1] = min(cap + ahead, 2 ** 31 - 1)
        got = attend(eng, q)
        there = eng.block_table.cpu().numpy().repeat(16, 1) >= 0      # (of the table's keys all that it has pages for)
        out, mag = reference(eng, [lens[0], cap, lens[2]], pars, q, ALL, 0, blocked=lambda b: ~there[b])
        assert ((got.double() - out).abs() <= bound(out, mag)).all()
    eng.close()


def test_plain_kernels_on_a_16_bit_cache():
    import paper_2508_18588_amd as hs
    eng, lens, pars, q = build((8, 2, 64), [0, 3], [100], [5, 60, 7], [1, 2, -4], seed=20)
    want = attend(eng, q)
    eng.set_flags(hs.HS_FLAG_REFERENCE_KERNELS)
    plain = attend(eng, q)
    check(plain, eng, lens, pars, q, ALL, 0)
    eng.set_flags(0)
    assert torch.equal(attend(eng, q), want)
    eng.close()


def test_refusals_from_python():
    eng, lens, pars, q = build((4, 2, 64), [0, 3], [64], [5, 6, 7], [1, 2, 1], seed=17)
    for off, pre in (([0], []), ([0, 3], [1, 2]), ([0, 2, 1], [1, 1]), ([0, 4], [1]), ([-1, 3], [1]), ([0, 3], [-1]), ([0, 3], [2 ** 31]), ([0, 1, 1, 2, 3], [1, 1, 1, 1])):
        with pytest.raises(ValueError):
            eng.set_shared_prefix(off, pre)
    with pytest.raises(ValueError):
        eng.attention_shared(0, q.float(), torch.zeros_like(q))
    with pytest.raises(ValueError):
        eng.attention_shared(0, q[:, :64], torch.zeros_like(q)[:, :64])
    with pytest.raises(ValueError):
        eng.attention_shared(0, q.cpu(), torch.zeros_like(q).cpu())
    eng.set_shared_prefix(None)
    with pytest.raises(ValueError):
        eng.attention_shared(0, q, torch.zeros_like(q))
    with pytest.raises(ValueError):
        eng.reserve(1)
    eng.close()
