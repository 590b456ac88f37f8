"""Log probabilities, entropies and largest alternatives against their definition in 64 bits.

What they may be off by: a weight's exponent d = (l - max) log2(e) / T has three roundings, which move the sum of weights by 3 * 2^-24 ln 2 of the average
|d|, at most log2(vocabulary) < 18; the exponential and 40 additions in 32 bits (32 of a lane, 6 of a wavefront, 2 of a workgroup) add 42 * 2^-24.  So ln S
is off by at most (3 * 18 * 0.7 + 42) 2^-24 < 5e-6, to which a result's own rounding comes; the sum of x exp(x), whose terms carry the same
errors times an |x| of 13 on average, by less than 1e-4."""
import numpy as np
import pytest
import torch

from window_common import engine, lay_out, chain

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def make(vocab, batch=1, nodes=1, **kw):
    return engine(1, 1, 64, [20] * batch, nodes, vocab=vocab, **kw)


def outputs(n, top, fill=5.0):
    f = lambda *s: torch.full(s, fill, device="cuda:0")
    out = dict(logprob=f(n), entropy=f(n))
    if top:
        out.update(top_token=torch.full((n, top), 77, device="cuda:0", dtype=torch.int32), top_logprob=f(n, top))
    return out


def logits_of(rows, vocab, seed, dtype=torch.float32, sharp=3.0, masked=0.0):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g, device="cuda:0") * sharp
    if masked:
        x.masked_fill_(torch.rand(rows, vocab, generator=g, device="cuda:0") < masked, -INF)
    return x.to(dtype)


def expect(x, tokens, temperature, top, rows=None):
    x = x.double()
    if rows is not None:
        x = x[rows.long()]
    lp = torch.log_softmax(x / temperature, -1)
    p = lp.exp()
    tok = tokens.long()
    inside = (tok >= 0) & (tok < x.shape[1])
    want = dict(logprob=torch.where(inside, lp.gather(1, tok.clamp(0, x.shape[1] - 1)[:, None])[:, 0], -INF),
                entropy=-torch.where(p > 0, p * lp, 0.0).sum(-1))
    if top:
        order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :top]
        want.update(top_token=order.int(), top_logprob=lp.gather(1, order))
    return want


def compare(got, want):
    for name in want:
        a, b = got[name].double(), want[name].double()
        if name == "top_token":
            assert torch.equal(got[name], want[name].int())
            continue
        assert torch.equal(torch.isnan(a), torch.isnan(b)), name
        ok = torch.isfinite(b)
        assert torch.equal(a[~ok & ~torch.isnan(b)], b[~ok & ~torch.isnan(b)]), name
        tol = (1e-4 if name == "entropy" else 5e-6) + 2.0 ** -24 * b[ok].abs()
        assert (tol - (a[ok] - b[ok]).abs()).min().item() >= 0 if ok.any() else True, (name, (a[ok] - b[ok]).abs().max().item())


def ask(eng, x, tokens, temperature=1.0, top=3, **kw):
    out = outputs(tokens.numel(), top)
    eng.logprobs(x, tokens, out, temperature, **kw)
    torch.cuda.synchronize()
    return out


def tokens_of(n, vocab, seed=1):
    return torch.as_tensor(np.random.default_rng(seed).integers(0, vocab, n), dtype=torch.int32, device="cuda:0")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,top", [(1, 1), (2, 2), (3, 0), (31, 31), (255, 5), (256, 32), (257, 3), (511, 32), (513, 1), (4096, 20), (8191, 7),
                                       (8192, 32), (8193, 8), (50001, 20), (151936, 32), (152064, 5)])
def test_against_the_definition(vocab, top, dtype):
    eng = make(vocab)
    x, tok = logits_of(5, vocab, vocab, dtype), tokens_of(5, vocab)
    for t in (1.0, 0.3, 2.5):
        compare(ask(eng, x, tok, t, top), expect(x, tok, float(np.float32(t)), top))
    eng.close()


@pytest.mark.parametrize("vocab", [600000, 1 << 21])
def test_vocabularies_beyond_the_units_in_lds(vocab):
    eng = make(vocab)
    x, tok = logits_of(3, vocab, 7), tokens_of(3, vocab)
    compare(ask(eng, x, tok, 0.9, 32), expect(x, tok, float(np.float32(0.9)), 32))
    eng.close()


def test_many_rows_in_several_launches():
    """More entries than the scratch holds at a time."""
    vocab = 40000
    eng = make(vocab)
    n = 30000
    x = logits_of(37, vocab, 3)
    rows = torch.as_tensor(np.random.default_rng(3).integers(0, 37, n), dtype=torch.int32, device="cuda:0")
    tok = tokens_of(n, vocab)
    got = ask(eng, x, tok, 1.0, 4, rows=rows)
    base = expect(x, torch.zeros(37, device="cuda:0"), 1.0, 4)
    lp = torch.log_softmax(x.double(), -1)
    want = {k: base[k][rows.long()] for k in base}
    want["logprob"] = lp[rows.long(), tok.long()]
    compare(got, want)
    eng.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_logits_take_the_lowest_token(dtype):
    vocab = 20000
    eng = make(vocab)
    x = torch.zeros(6, vocab, device="cuda:0")
    x[1] = -3.0
    x[2, ::7] = 1.0
    x[3, 300:] = 2.0
    x[4] = torch.arange(vocab, device="cuda:0") % 5
    x[5, ::2] = -0.0                              # (0 and -0 are equal)
    x, tok = x.to(dtype), tokens_of(6, vocab)
    compare(ask(eng, x, tok, 1.0, 32), expect(x, tok, 1.0, 32))
    eng.close()


@pytest.mark.parametrize("crowd", [40, 300, 2000, 9000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_crowded_units(crowd, dtype):
    """The largest logits lie together in fewer units than are looked for, and more of them than there is room for at a time; and one of them in
    every unit."""
    vocab = 60000
    eng = make(vocab)
    x = logits_of(4, vocab, crowd, torch.float32, 1.0)
    x[0, 1000:1000 + crowd] += 30
    x[1, vocab - crowd:] += 30
    x[2, ::max(1, vocab // crowd)] += 30
    x[3, 5:5 + crowd] = 40 + torch.arange(crowd, device="cuda:0") % 3
    x, tok = x.to(dtype), tokens_of(4, vocab)
    for top in (1, 20, 32):
        compare(ask(eng, x, tok, 1.0, top), expect(x, tok, 1.0, top))
    eng.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_excluded_tokens(dtype):
    vocab = 9000
    eng = make(vocab)
    x = logits_of(8, vocab, 5, dtype, masked=0.5)
    x[1] = -INF
    x[1, 4321] = 2.0                              # one token is left
    x[2] = -INF
    x[2, [5, 8999]] = 1.0
    x[3, 300:] = -INF
    x[4, :8900] = -INF
    x[5, 8192:] = -INF                            # a whole chunk
    tok = torch.tensor([3, 4321, 5, 10, 8950, 8500, -1, vocab], dtype=torch.int32, device="cuda:0")
    want = expect(x, tok, 1.0, 20)
    compare(ask(eng, x, tok, 1.0, 20), want)
    eng.close()


def test_rows_of_nothing_and_rows_of_nan():
    vocab = 9000
    eng = make(vocab)
    x = logits_of(6, vocab, 6)
    x[0] = -INF
    x[1, 77] = NAN
    x[2, 8999] = INF
    x[3] = -INF
    x[3, 5] = NAN
    tok = torch.tensor([1, 2, 3, 4, 5, 6], dtype=torch.int32, device="cuda:0")
    out = ask(eng, x, tok, 1.0, 3)
    assert out["logprob"][0] == -INF and out["entropy"][0] == 0 and out["top_token"][0].tolist() == [0, 1, 2] and (out["top_logprob"][0] == -INF).all()
    for i in (1, 2, 3):
        assert torch.isnan(out["logprob"][i]) and torch.isnan(out["entropy"][i])
        assert (out["top_token"][i] == -1).all() and torch.isnan(out["top_logprob"][i]).all()
    compare({k: v[4:] for k, v in out.items()}, expect(x[4:], tok[4:], 1.0, 3))
    eng.close()


def test_extreme_logits_and_temperatures():
    vocab = 3001
    eng = make(vocab)
    x = logits_of(4, vocab, 8) * 1e4
    x[1] = 3e38 * torch.sign(x[1])
    x[2] = 1e-30 * x[2]
    tok = tokens_of(4, vocab)
    for t in (1.0, 1e-20, 1e20):
        got = ask(eng, x, tok, t, 5)
        want = expect(x, tok, float(np.float32(t)), 5)
        keep = torch.isfinite(want["logprob"]) & (want["logprob"] > -1e30)
        assert torch.equal(got["top_token"], want["top_token"])
        d = (got["logprob"].double() - want["logprob"])[keep].abs()
        assert (d <= 5e-6 + 2.0 ** -23 * want["logprob"][keep].abs()).all()
        assert ((got["entropy"].double() - want["entropy"]).abs() < 1e-4).all()
    eng.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_alignment_rows_and_live(dtype):
    vocab = 5003
    eng = make(vocab)
    wide = logits_of(9, vocab + 14, 9, dtype)
    x = wide[:, 1:vocab + 1]                      # rows that begin anywhere
    x[:, :] = x.clone()
    rows = torch.tensor([8, 0, 0, 3, -1, 9, 2 ** 31 - 1, 4], dtype=torch.int32, device="cuda:0")
    tok = tokens_of(8, vocab)
    out = ask(eng, x, tok, 1.0, 4, rows=rows)
    good = torch.tensor([0, 1, 2, 3, 7], device="cuda:0")
    compare({k: v[good] for k, v in out.items()}, expect(x, tok[good], 1.0, 4, rows[good]))
    for i in (4, 5, 6):
        assert torch.isnan(out["logprob"][i]) and torch.isnan(out["entropy"][i]) and (out["top_token"][i] == -1).all()
    one = outputs(8, 2)
    eng.logprobs(x, tok, one, live=torch.tensor([3], dtype=torch.int32, device="cuda:0"))
    compare({k: v[:3] for k, v in one.items()}, expect(x[:3], tok[:3], 1.0, 2))
    assert (one["logprob"][3:] == 5).all() and (one["top_token"][3:] == 77).all()
    alone = dict(logprob=torch.zeros(8, device="cuda:0"))
    eng.logprobs(x, tok, alone)
    assert torch.equal(alone["logprob"], ask(eng, x, tok, 1.0, 0)["logprob"])
    eng.close()


def test_bits_do_not_depend_on_what_else_is_asked():
    vocab = 30011
    eng = make(vocab)
    x, tok = logits_of(40, vocab, 10), tokens_of(40, vocab)
    full = ask(eng, x, tok, 0.8, 6)
    for i in (0, 17, 39):
        one = ask(eng, x[i:i + 1], tok[i:i + 1], 0.8, 6)
        assert all(torch.equal(one[k][0], full[k][i]) for k in one)
    assert torch.equal(ask(eng, x, tok, 0.8, 0)["logprob"], full["logprob"])
    eng.close()


@pytest.mark.parametrize("given", [False, True])
def test_emitted_tokens(given):
    vocab, B, k = 4999, 5, 4
    eng = make(vocab, B, k + 1)
    x = logits_of(B * (k + 1), vocab, 11, torch.bfloat16 if given else torch.float32)
    lay_out(eng, [20] * B, [chain(k), None, chain(k), chain(0), chain(2)])
    counts = np.asarray([3, 0, 5, 1, 2])
    path = np.asarray([[0, 1, 2, 0, 0], [9, 9, 9, 9, 9], [0, 1, 2, 3, 4], [0] * 5, [0, 2, 0, 0, 0]])
    toks = np.random.default_rng(4).integers(0, vocab, (B, k + 1))
    i32 = lambda a: torch.as_tensor(a, dtype=torch.int32, device="cuda:0")
    eng.st["n_out"].copy_(i32(counts)), eng.st["path_row"].copy_(i32(path)), eng.st["out_tok"].copy_(i32(toks))
    out = outputs(B * (k + 1), 3)
    if given:
        eng.emitted_logprobs(out, 0.7, logits=x)
    else:
        eng.logits = x
        eng._structs()
        eng.emitted_logprobs(out, 0.7)
    off = eng.st["row_off"].cpu().numpy()
    for b in range(B):
        for i in range(k + 1):
            e = b * (k + 1) + i
            if i >= counts[b]:
                assert out["logprob"][e] == 5 and (out["top_token"][e] == 77).all()
                continue
            want = expect(x[off[b] + path[b, i]][None], i32([toks[b, i]]), float(np.float32(0.7)), 3)
            compare({n: t[e:e + 1] for n, t in out.items()}, want)
    eng.close()


def test_captured_and_replayed():
    vocab = 12000
    eng = make(vocab)
    x, tok, out = logits_of(6, vocab, 12), tokens_of(6, vocab), outputs(6, 5)
    eng.logprobs(x, tok, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        eng.logprobs(x, tok, out)
    for seed in (13, 14, 15):
        x.copy_(logits_of(6, vocab, seed))
        tok.copy_(tokens_of(6, vocab, seed))
        g.replay()
        torch.cuda.synchronize()
        compare(out, expect(x, tok, 1.0, 5))
        again = ask(eng, x, tok, 1.0, 5)
        assert all(torch.equal(again[n], out[n]) for n in out)
    eng.close()


def test_refusals_from_python():
    vocab = 1000
    eng = make(vocab)
    x, tok = logits_of(4, vocab, 16), tokens_of(4, vocab)
    good = outputs(4, 2)
    bad = [dict(), dict(entropy=good["entropy"]), dict(logprob=good["logprob"].double()), dict(logprob=good["logprob"][:3]),
           dict(logprob=good["logprob"], top_token=good["top_token"]), dict(logprob=good["logprob"], other=good["entropy"]),
           dict(logprob=good["logprob"], top_token=good["top_token"][:3], top_logprob=good["top_logprob"][:3]),
           dict(logprob=good["logprob"].cpu())]
    for out in bad:
        with pytest.raises(ValueError):
            eng.logprobs(x, tok, out)
    for args in ((x[:3], tok), (x[:, :999], tok), (x.half(), tok), (x, tok.long()), (x.t(), tok), (x, tok.cpu())):
        with pytest.raises(ValueError):
            eng.logprobs(*args, good)
    with pytest.raises(ValueError):
        eng.logprobs(x, tok, good, rows=tok[:2])
    eng.logprobs(x, tok[:0], outputs(0, 0) | dict(logprob=good["logprob"]))
    eng.close()
