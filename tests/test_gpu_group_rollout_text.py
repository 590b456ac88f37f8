"""Every token of a forked rollout against its own text: an engine without shared pages or prefixes computes the logits from prompt and tokens anew.

What the two passes may differ by: E = 0.02 in a logit (the tolerance of the path).  A greedy token was the largest in one pass, so it is at most 2 E below
the largest in the other.  A log probability l - ln sum exp(l) moves by E, and by E again through the sum.  The entropy's derivative along a
change of logits d, |d| <= E, is -sum p (ln p + H) d, at most E sqrt(var ln p); on the way ln p moves by at most 2 E and the weights by factors of
at most exp(2 E), so that sqrt(var) stays below exp(E) (sqrt(var of the reference) + 2 E).  To that come 5e-6 and 1e-4 of the 32-bit sums (test_gpu_logprobs)."""
import numpy as np
import pytest
import torch

from test_gpu_group_rollout import GROUPS, MEMBERS, N, engine, model, roll, start_forked  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu
E, B, STEP = 0.02, GROUPS * MEMBERS, 4


def logits_of_texts(ref, prompts, toks):
    """[B, N, vocab] in 64 bits: row i decides on token i of toks[b] behind prompts[b]."""
    parts = []
    for i in range(0, N, STEP):
        texts = [np.concatenate([prompts[b], toks[b][:i]]).astype(np.int32) for b in range(B)]
        ref.load_sequences(texts, [N] * B)
        ref.prefill_chunked(64)
        m = ref.set_rows([dict(tok=np.concatenate([x[-1:], toks[b][i:i + STEP - 1]]).astype(np.int32), parent=np.arange(-1, STEP - 1),
                               pos=len(x) - 1 + np.arange(STEP)) for b, x in enumerate(texts)])
        ref.verify()
        torch.cuda.synchronize()
        assert ref.poll_error() == 0
        parts.append(ref.logits[:m].view(B, STEP, -1).double().clone())
    return torch.cat(parts, 1)


def within(x, toks, lps, ents):
    """Which tokens, log probabilities and entropies are within their bounds of the logits x."""
    tok = torch.as_tensor(np.asarray(toks), device="cuda:0")[..., None]
    lp = torch.log_softmax(x, -1)
    p = lp.exp()
    H = -(p * lp).sum(-1)
    spread = (p * (lp + H[..., None]) ** 2).sum(-1).sqrt()
    f64 = lambda a: torch.as_tensor(np.asarray(a), dtype=torch.float64, device="cuda:0")
    return (x.amax(-1) - x.gather(2, tok)[..., 0] <= 2 * E, (lp.gather(2, tok)[..., 0] - f64(lps)).abs() <= 2 * E + 5e-6,
            (H - f64(ents)).abs() <= E * np.exp(E) * (spread + 2 * E) + 1e-4)


def test_every_token_is_the_one_of_its_text(model):  # noqa: F811
    shape, w, rope, prompts = model
    ref, first = engine(model), None
    per = [prompts[b // MEMBERS] for b in range(B)]
    # the same text with another page of the prompt: the bounds tell them apart
    other = [np.concatenate([p[:16], prompts[(b // MEMBERS + 1) % GROUPS][16:32], p[32:]]) for b, p in enumerate(per)]
    for turn in range(2):      # without drafts, and with drafts from texts that are half right
        eng = engine(model, pages=60)
        start_forked(eng, prompts)
        toks, lps, ents, steps = roll(eng, prompts, shape.vocab, first, True)
        eng.close()
        assert all(len(t) == N for t in toks)
        for ok in within(logits_of_texts(ref, per, toks), toks, lps, ents):
            assert ok.all()
        token, lp, _ = within(logits_of_texts(ref, other, toks), toks, lps, ents)
        assert token.float().mean() < 0.5 and lp.float().mean() < 0.5
        first = toks
    ref.close()
