"""Log probabilities of what a step emits with every kind of acceptance, and questions about nothing."""
import numpy as np
import pytest
import torch

from hs_inputs import history_with_context
from test_gpu_group_rollout import GROUPS, MEMBERS, engine, model, start_alone  # noqa: F401  (the fixture)
from test_gpu_logprobs import compare, expect, logits_of, make, tokens_of

pytestmark = pytest.mark.gpu
SHARP = 0.02      # the temperature of acceptance: this model's logits differ by a few tenths, and drafts are to be accepted now and then


@pytest.mark.parametrize("rows", [0, 4])
@pytest.mark.parametrize("top", [0, 3])
def test_no_tokens(rows, top):
    """Nothing is asked: outputs of size 0 (whose address is none) are as good as others, and so are logits of no rows."""
    eng = make(1000)
    x, none = logits_of(rows, 1000, 1), torch.zeros(0, dtype=torch.int32, device="cuda:0")
    out = dict(logprob=torch.zeros(0, device="cuda:0"), entropy=torch.zeros(0, device="cuda:0"))
    if top:
        out.update(top_token=torch.zeros(0, top, dtype=torch.int32, device="cuda:0"), top_logprob=torch.zeros(0, top, device="cuda:0"))
    eng.logprobs(x, none, out)
    eng.logprobs(x, none, out, rows=none, live=torch.zeros(1, dtype=torch.int32, device="cuda:0"))
    torch.cuda.synchronize()
    assert eng.poll_error() == 0
    eng.close()


@pytest.mark.parametrize("how", ["greedy", "rejection", "given"])
def test_emitted_tokens_of_steps(model, how):  # noqa: F811
    """With drafts that are chains the i-th emitted token was decided in the sequence's i-th row, whoever decided."""
    from paper_2508_18588_amd import HS_ACCEPT_GREEDY, HS_ACCEPT_REJECTION
    from paper_2508_18588_amd.runtime import Policy
    shape, w, rope, prompts = model
    B, pol, T = GROUPS * MEMBERS, Policy(window=8, m_min=2, k_fixed=4, k_max=4), float(np.float32(0.8))
    eng = engine(model)
    start_alone(eng, prompts)
    rng, g = np.random.default_rng(1), torch.Generator(device="cuda:0").manual_seed(1)
    # histories whose next tokens are the greedy ones, as far as they are known: a first rollout of a few steps
    eng.set_history([[np.zeros(4, np.int32)]] * B)
    first = [[] for _ in range(B)]
    for _ in range(8):
        eng.step(pol)
        for b, (n, t) in enumerate(zip(eng.st["n_out"].tolist(), eng.st["out_tok"].tolist())):
            first[b] += t[:n]
    start_alone(eng, prompts)
    eng.set_history([[history_with_context(prompts[b // MEMBERS], np.asarray(first[b], np.int32), 8)] for b in range(B)])
    out = dict(logprob=torch.zeros(B * 5, device="cuda:0"), entropy=torch.zeros(B * 5, device="cuda:0"),
               top_token=torch.zeros(B * 5, 3, dtype=torch.int32, device="cuda:0"), top_logprob=torch.zeros(B * 5, 3, device="cuda:0"))
    several, p = 0, torch.zeros_like(eng.logits)
    for step in range(5):
        eng.draft(pol)
        eng.verify()
        if how == "given":
            eng.probs(eng.logits, p, SHARP, live=True)
            eng.accept_probs(p, None, torch.rand(eng.max_rows, generator=g, device="cuda:0"), torch.rand(B, generator=g, device="cuda:0"))
        elif how == "rejection":
            eng.accept(HS_ACCEPT_REJECTION, SHARP, int(rng.integers(1 << 30)))
        else:
            eng.accept(HS_ACCEPT_GREEDY)
        for t in out.values():
            t.fill_(5)
        eng.emitted_logprobs(out, T)
        torch.cuda.synchronize()
        n_out, tok, off = eng.st["n_out"].tolist(), eng.st["out_tok"], eng.st["row_off"].tolist()
        for b in range(B):
            n = n_out[b]
            assert min(1, off[b + 1] - off[b]) <= n <= off[b + 1] - off[b]      # (none when the budget is used up)
            several += n > 1
            rows = torch.arange(off[b], off[b] + n, device="cuda:0")
            compare({k: t[b * 5:b * 5 + n] for k, t in out.items()}, expect(eng.logits, tok[b, :n], T, 3, rows))
            assert all((t[b * 5 + n:b * 5 + 5] == 5).all() for t in out.values())
        eng.commit(pol)
    assert several > 0      # (drafts were accepted)
    eng.close()
