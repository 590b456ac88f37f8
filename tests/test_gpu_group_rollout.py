"""A rollout of groups of responses with the operators together: prompts computed once, forked, decoded with drafts while the prompts' keys are read
once per group, pages reserved on the way and compacted in between, log probabilities of what was emitted -- against the same rollout of sequences
that hold everything for themselves."""
import numpy as np
import pytest
import torch

from hs_inputs import CONFIG_SHAPES, history_with_context, make_prompts, make_weights, mutate, rope_table

pytestmark = pytest.mark.gpu
GROUPS, MEMBERS, N = 2, 3, 12


@pytest.fixture(scope="module")
def model():
    shape = CONFIG_SHAPES[1]
    return shape, make_weights(shape, 1), rope_table(512, shape.head_dim), make_prompts(GROUPS, 90, shape.vocab, seed=6)


def engine(model, **kw):
    from paper_2508_18588_amd.runtime import Engine
    shape, w, rope, prompts = model
    return Engine(shape, w, rope, max_batch=GROUPS * MEMBERS, k_max=4, c_max=1, max_len=420, max_rows=128, **kw)


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda:0")


def start_alone(eng, prompts):
    eng.load_sequences([p for p in prompts for _ in range(MEMBERS)], [N] * GROUPS * MEMBERS)
    eng.prefill_chunked(64)


def start_forked(eng, prompts):
    """The first sequence of each group has the prompt; the others take its text."""
    one = np.zeros(1, np.int32)
    eng.load_sequences([p if i == 0 else one for p in prompts for i in range(MEMBERS)], [N] * GROUPS * MEMBERS)
    eng.reserve(0, first=torch.zeros(GROUPS * MEMBERS, dtype=torch.int32, device="cuda:0"))
    eng.prefill_chunked(64)
    eng.fork(i32([g * MEMBERS for g in range(GROUPS) for _ in range(MEMBERS)]))
    eng.set_shared_prefix(np.arange(0, GROUPS * MEMBERS + 1, MEMBERS), [(len(p) - 1) // 16 * 16 for p in prompts])


def roll(eng, prompts, vocab, first, pooled):
    """Greedy rollout with drafts from texts that are half right; returns tokens, log probabilities, and the number of steps."""
    from paper_2508_18588_amd.runtime import Policy
    B, pol = GROUPS * MEMBERS, Policy(window=8, m_min=3, k_fixed=4, k_max=4)
    rng = np.random.default_rng(5)
    if first is None:
        cands = [[np.zeros(4, np.int32)]] * B
    else:
        cands = [[history_with_context(prompts[b // MEMBERS], mutate(np.asarray(first[b], np.int32), 0.3, 0.0, vocab, rng), 8)] for b in range(B)]
    eng.set_history(cands)
    toks, lps, ents, steps = [[] for _ in range(B)], [[] for _ in range(B)], [[] for _ in range(B)], 0
    out = dict(logprob=torch.zeros(B * 5, device="cuda:0"), entropy=torch.zeros(B * 5, device="cuda:0"),
               top_token=torch.zeros(B * 5, 2, dtype=torch.int32, device="cuda:0"), top_logprob=torch.zeros(B * 5, 2, device="cuda:0"))
    while min(len(t) for t in toks) < N and steps < 2 * N:
        if pooled:
            eng.reserve(5)
            if steps % 3 == 2:
                eng.compact()
        eng.step(pol)
        eng.emitted_logprobs(out)
        torch.cuda.synchronize()
        assert eng.poll_error() == 0
        n, tok = eng.st["n_out"].cpu().numpy(), eng.st["out_tok"].cpu().numpy()
        for b in range(B):
            for i in range(n[b]):
                e = b * 5 + i
                toks[b].append(int(tok[b, i]))
                lps[b].append(out["logprob"][e].item())
                ents[b].append(out["entropy"][e].item())
                assert out["top_token"][e, 0].item() == tok[b, i]      # greedy: the token is the largest one
                assert out["top_logprob"][e, 0].item() == lps[b][-1] and out["top_logprob"][e, 1] <= out["top_logprob"][e, 0]
        steps += 1
    return toks, lps, ents, steps


def test_forked_rollout_is_the_rollout_of_separate_sequences(model):
    shape, w, rope, prompts = model
    alone = engine(model)
    start_alone(alone, prompts)
    t0, l0, e0, s0 = roll(alone, prompts, shape.vocab, None, False)
    alone.close()
    runs = []
    for first in (None, t0):
        eng = engine(model, pages=60, shuffle_pages_seed=None)
        start_forked(eng, prompts)
        held = int((eng.page_refs > 0).sum())
        full = sum((len(p) - 1) // 16 for p in prompts)
        assert held <= full + 2 * GROUPS * MEMBERS and (eng.page_refs == MEMBERS).sum().item() == full
        runs.append(roll(eng, prompts, shape.vocab, first, True))
        # everything is given back
        B = GROUPS * MEMBERS
        eng.free_pages(i32([0] * B), i32([2 ** 31 - 1] * B))
        assert eng.compact().item() == 0 and (eng.page_refs == 0).all() and (eng.block_table == -1).all()
        eng.close()
    for toks, lps, ents, steps in runs:
        for b in range(GROUPS * MEMBERS):
            # (bf16 activations in another order of sums: logits may differ by 0.02, the fixed tolerance of the path; a rollout whose two largest
            # logits come nearer than that somewhere may part there)
            n = next((i for i in range(N) if toks[b][i] != t0[b][i]), N)
            assert n >= 1
            if n < N:
                assert abs(lps[b][n] - l0[b][n]) < 0.08
            for i in range(n):
                assert abs(lps[b][i] - l0[b][i]) < 0.08 and abs(ents[b][i] - e0[b][i]) < 0.4
    assert runs[1][3] < runs[0][3]      # drafts were accepted
    # responses of a group start with the same text and, greedily, are the same
    for g in range(GROUPS):
        assert all(runs[0][0][g * MEMBERS] == runs[0][0][g * MEMBERS + i] for i in range(MEMBERS))


def test_verify_with_shared_prefixes(model):
    """Logits of one pass with prefixes shared and read per sequence, on the same cache; with the plain kernels the same bits."""
    import paper_2508_18588_amd as hs
    shape, w, rope, prompts = model
    eng = engine(model, pages=60)
    start_forked(eng, prompts)
    eng.reserve(5)
    rng = np.random.default_rng(3)
    rows = [dict(tok=rng.integers(0, shape.vocab, n), parent=np.arange(-1, n - 1), pos=len(prompts[b // MEMBERS]) - 1 + np.arange(n))
            for b, n in enumerate([1, 5, 3, 2, 1, 4])]
    m = eng.set_rows(rows)

    def logits():
        eng.verify()
        torch.cuda.synchronize()
        assert eng.poll_error() == 0
        return eng.logits[:m].clone()
    shared = logits()
    off, pre = np.arange(0, GROUPS * MEMBERS + 1, MEMBERS), [(len(p) - 1) // 16 * 16 for p in prompts]
    eng.set_shared_prefix(None)
    alone = logits()
    assert not torch.equal(shared, alone)                  # (it did run)
    assert (shared - alone).abs().max() < 2e-2             # (the tolerance of the path)
    eng.set_flags(hs.HS_FLAG_REFERENCE_KERNELS)
    plain = logits()
    eng.set_shared_prefix(off, pre)
    assert torch.equal(logits(), plain)
    eng.set_flags(0)
    assert torch.equal(logits(), shared)
    # layers with a window read every sequence's own table
    eng.set_window([40, 0], 4)
    half = logits()
    eng.set_shared_prefix(None)
    assert (logits() - half).abs().max() < 2e-2
    eng.set_window(None)
    eng.close()


def test_captured_step_of_a_forked_rollout(model):
    """draft, verify with shared prefixes, accept + commit and the log probabilities in a graph, against eager steps."""
    from paper_2508_18588_amd.runtime import Policy
    shape, w, rope, prompts = model
    B, pol = GROUPS * MEMBERS, Policy(window=8, m_min=3, k_fixed=4, k_max=4)
    results = []
    for captured in (False, True):
        eng = engine(model, pages=60)
        start_forked(eng, prompts)
        eng.set_history([[np.zeros(4, np.int32)]] * B)
        out = dict(logprob=torch.zeros(B * 5, device="cuda:0"))

        def step():
            eng.reserve(5)
            eng.step(pol)
            eng.emitted_logprobs(out)
        step()
        torch.cuda.synchronize()
        if captured:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
        seen = []
        for _ in range(4):
            g.replay() if captured else step()
            torch.cuda.synchronize()
            seen.append((eng.st["out_tok"].clone(), out["logprob"].clone(), eng.block_table.clone(), eng.seq_len.clone()))
        assert eng.poll_error() == 0
        results.append(seen)
        eng.close()
    for a, b in zip(*results):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
