"""Shared prefixes borrow idle arrays of the workspace: what a step leaves there for its caller stays as it is, and log probabilities may run beside
the next step."""
import numpy as np
import pytest
import torch

from test_gpu_group_rollout import engine, model, start_forked  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def test_a_steps_views_and_logits_stay(model):  # noqa: F811
    """The debug views and the logits that the workspace keeps, before and after attention with shared prefixes and log probabilities of many rows;
    and the next step on the same cache has the same bits."""
    shape, w, rope, prompts = model
    eng = engine(model, pages=60, keep_logits=False, workspace_logits=True)
    start_forked(eng, prompts)
    eng.reserve(5)
    rng = np.random.default_rng(3)
    m = eng.set_rows([dict(tok=rng.integers(0, shape.vocab, n), parent=np.arange(-1, n - 1), pos=len(prompts[b // 3]) - 1 + np.arange(n))
                      for b, n in enumerate([1, 5, 3, 2, 1, 4])])

    def views():
        torch.cuda.synchronize()
        return [eng.debug_tensor(i).clone() for i in range(6)]
    eng.verify()
    first = views()
    q = torch.randn(m, shape.n_q_heads * shape.head_dim, device="cuda:0").to(torch.bfloat16)
    for layer in range(eng.n_layers):
        eng.attention_shared(layer, q, torch.empty_like(q))
    n = 3000
    x = torch.randn(40, shape.vocab, device="cuda:0")
    tok = torch.arange(n, dtype=torch.int32, device="cuda:0") % shape.vocab
    out = dict(logprob=torch.zeros(n, device="cuda:0"), top_token=torch.zeros(n, 4, dtype=torch.int32, device="cuda:0"),
               top_logprob=torch.zeros(n, 4, device="cuda:0"))
    eng.logprobs(x, tok, out, rows=tok % 40)
    assert all(torch.equal(a, b) for a, b in zip(first, views()))
    eng.verify()
    assert all(torch.equal(a, b) for a, b in zip(first, views()))
    eng.close()


def test_log_probabilities_beside_the_next_step(model):  # noqa: F811
    """On a stream of their own, of logits that the caller keeps: they and the step have the same bits as one after the other."""
    shape, w, rope, prompts = model
    eng = engine(model, pages=60)
    start_forked(eng, prompts)
    eng.reserve(5)
    eng.set_rows([dict(tok=np.arange(5), parent=np.arange(-1, 4), pos=len(prompts[b // 3]) - 1 + np.arange(5)) for b in range(6)])
    n = 3000
    x = torch.randn(40, shape.vocab, device="cuda:0")
    tok = torch.arange(n, dtype=torch.int32, device="cuda:0") % shape.vocab
    rows = tok % 40
    outs = [dict(logprob=torch.zeros(n, device="cuda:0"), entropy=torch.zeros(n, device="cuda:0"),
                 top_token=torch.zeros(n, 4, dtype=torch.int32, device="cuda:0"), top_logprob=torch.zeros(n, 4, device="cuda:0")) for _ in range(2)]
    eng.verify()
    eng.logprobs(x, tok, outs[0], rows=rows)
    torch.cuda.synchronize()
    want, side = eng.logits.clone(), torch.cuda.Stream()
    for _ in range(5):
        eng.logits.zero_()
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(4):
            with torch.cuda.stream(side):
                eng.logprobs(x, tok, outs[1], rows=rows)
            eng.verify()
        torch.cuda.synchronize()
        assert torch.equal(eng.logits, want) and all(torch.equal(outs[0][k], outs[1][k]) for k in outs[0])
    eng.close()
