"""hs_probs and hs_accept_probs against their definitions in 64 bits: chains, trees, drafts with and without a distribution, odd
vocabularies and strides, probabilities that are none, random numbers at the ends of their range; the distribution of what is
emitted; and the whole of a sampled step, against hs_accept with the same random numbers."""
import numpy as np
import pytest
import torch

from window_common import chain, depths, engine, random_tree

pytestmark = pytest.mark.gpu


def _probs_engine(vocab, rows, **kw):
    return engine(1, 1, 64, [8] * rows, 1, vocab=vocab, **kw)


# ---------------------------------------------------------------- probabilities

def _check_probs(got, x, temperature, dst):
    x = x.double()
    top = x.amax(-1, keepdim=True)
    e = torch.exp((x - top) / temperature)
    want = e / e.sum(-1, keepdim=True)
    err = (got.double() - want).abs()
    # 32-bit exponents, exponentials and sums: their exponential, a product and a quotient are off by a few units of 2^-24 each, the
    # sum of up to 2^18 positive terms by less than 40 (a tree of partial sums of at most 300 terms in a row), and l - max is rounded
    # once: 2^-24 |l - max| / T in the exponent.  Values below 2^-126 may vanish.
    tol = want * (2.0 ** -24 * (60 + 2 * ((top - x) / temperature).clamp(max=200)))
    if dst == torch.bfloat16:
        tol = tol + 2.0 ** -8 * want
    assert (err <= tol + 2.0 ** -125).all(), (err - tol).max()


@pytest.mark.parametrize("src,dst", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32),
                                     (torch.bfloat16, torch.bfloat16)])
@pytest.mark.parametrize("vocab,rows,pad", [(1, 3, 0), (7, 5, 1), (1000, 1, 0), (4096, 9, 8), (5003, 33, 4), (65537, 2, 3), (151936, 3, 0)])
def test_probs(src, dst, vocab, rows, pad):
    eng = _probs_engine(vocab, rows)
    g = torch.Generator(device="cuda:0").manual_seed(vocab)
    x = (torch.randn(rows + 1, vocab + pad, generator=g, device="cuda:0") * 4 - 30).to(src)
    out = torch.full((rows + 1, vocab + 2 * pad), 7.0, device="cuda:0", dtype=dst)
    for t in (1.0, 0.05, 30.0):
        eng.probs(x[:rows], out, t)
        _check_probs(out[:rows, :vocab], x[:rows, :vocab], t, dst)
    assert (out[rows] == 7.0).all() and (out[:, vocab:] == 7.0).all()
    eng.close()


@pytest.mark.parametrize("rows", [1, 7, 64, 257, 700])
def test_probs_for_few_and_many_rows(rows):
    """Whatever shape a launch takes: every row, and no row beyond the live ones."""
    vocab = 20011
    eng = engine(1, 1, 64, [8] * 4, 1, vocab=vocab, max_rows=512)
    g = torch.Generator(device="cuda:0").manual_seed(rows)
    x = torch.randn(rows, vocab, generator=g, device="cuda:0") * 5
    out = torch.full((rows, vocab), 7.0, device="cuda:0")
    eng.probs(x, out, 0.8)
    _check_probs(out, x, 0.8, torch.float32)
    out.fill_(7.0)
    eng.st["row_off"][4] = rows // 2
    eng.probs(x, out, 0.8, live=True)
    _check_probs(out[:rows // 2], x[:rows // 2], 0.8, torch.float32)
    assert (out[rows // 2:] == 7.0).all()
    eng.st["row_off"][4] = rows + 5                    # (more than the arrays have)
    eng.probs(x, x, 0.8, live=True)                    # in place
    out.fill_(7.0)
    eng.st["row_off"][4] = 0
    eng.probs(x, out, 0.8, live=True)
    assert (out == 7.0).all()
    assert (x.sum(-1) - 1.0).abs().max() < 1e-5
    eng.close()


def test_a_rows_probabilities_do_not_depend_on_the_other_rows():
    """The same bits whether a row is one of 330 of 600 KB, which a workgroup each takes, or of a few."""
    vocab, rows = 151936, 330
    eng = engine(1, 1, 64, [8] * 4, 1, vocab=vocab)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    x = torch.randn(rows, vocab, generator=g, device="cuda:0") * 4
    x[::7, 5000:5100] = -float("inf")
    out, few = (torch.zeros(rows, vocab, device="cuda:0") for _ in range(2))
    eng.probs(x, out, 0.9)
    _check_probs(out[::40], x[::40], 0.9, torch.float32)
    for r, n in ((0, 1), (100, 3), (200, 64), (329, 1)):
        eng.probs(x[r:r + n], few[r:r + n], 0.9)
        assert torch.equal(few[r:r + n], out[r:r + n])
    eng.close()


def test_probs_of_many_short_rows():
    vocab, rows = 100, 300001                          # more units of a softmax than there is room for at a time
    eng = engine(1, 1, 64, [8] * 4, 1, vocab=vocab)
    x = torch.randn(rows, vocab, device="cuda:0")
    out = torch.zeros(rows, vocab, device="cuda:0")
    eng.probs(x, out, 1.0)
    for r in (0, 262140, 300000):
        _check_probs(out[r:r + 10], x[r:r + 10], 1.0, torch.float32)
    assert (out.sum(-1) - 1.0).abs().max() < 1e-5
    eng.close()


@pytest.mark.parametrize("rows", [3, 600])
def test_probs_of_excluded_and_odd_logits(rows):
    vocab, inf, nan = 10000, float("inf"), float("nan")
    eng = engine(1, 1, 64, [8] * 4, 1, vocab=vocab, max_rows=rows)
    x = torch.randn(rows, vocab, device="cuda:0")
    x[0, :9999] = -inf                                 # one token left
    x[1] = -inf                                        # none
    x[2, 5000:] = -inf
    out = torch.full((rows, vocab), 7.0, device="cuda:0")
    eng.probs(x, out, 0.5)
    assert (out[0, :9999] == 0).all() and out[0, 9999] == 1.0
    assert (out[1] == 0).all()
    assert (out[2, 5000:] == 0).all() and (out[2].sum() - 1.0).abs() < 1e-5
    x[0, 17], x[1, 9000], x[2, 0] = nan, inf, torch.finfo(torch.float32).min
    eng.probs(x, out, 0.5)
    assert torch.isnan(out[0]).all() and torch.isnan(out[1, 9000]) and out[2, 0] == 0
    x[2] = torch.finfo(torch.float32).min              # a mask of the type's lowest value on every token: all alike
    eng.probs(x, out, 0.5)
    assert (out[2] - 1.0 / vocab).abs().max() < 1e-8
    # the ends of the temperature's range: the largest logit alone, and all that are not excluded alike
    x = torch.randn(rows, vocab, device="cuda:0")
    x[:, 100:200] = -inf
    eng.probs(x, out, 1e-45)
    assert (out.argmax(-1) == x.argmax(-1)).all() and (out.sum(-1) == 1.0).all() and (out.amax(-1) == 1.0).all()
    eng.probs(x, out, inf)
    assert (out[:, 100:200] == 0).all() and (out[:, 200:] - 1.0 / (vocab - 100)).abs().max() < 1e-8
    eng.close()


# ---------------------------------------------------------------- verification

def definition(pars, toks, p, q, ua, us, width):
    """Acceptance in 64 bits.  p, q: [rows, vocab] as numpy float64, what does not count already 0."""
    V, r0, out = p.shape[1], 0, dict(accept_len=[], n_out=[], out_tok=[], path_row=[])
    for b, par in enumerate(pars):
        if par is None:
            out["accept_len"].append(0); out["n_out"].append(0)
            out["out_tok"].append([-9] * width); out["path_row"].append([-9] * width)
            continue
        cur, toks_b, path, done = 0, [], [0], False
        while not done:
            w, z, done = p[r0 + cur], 1.0, True
            if len(path) < width:
                for c in [i for i in range(1, len(par)) if par[i] == cur]:
                    t = int(toks[b][c])
                    known = 0 <= t < V
                    qt = (1.0 if q is None else q[r0 + cur, t]) if known else 0.0
                    if ua[r0 + c] * z * qt < (w[t] if known else 0.0):
                        cur, done = c, False
                        toks_b.append(t); path.append(c)
                        break
                    if q is None:
                        w = w.copy()
                        if known:
                            w[t] = 0.0
                    else:
                        w = np.maximum(w - z * q[r0 + cur], 0.0)
                    z = w.sum()
        if not w.sum() > 0:
            w = p[r0 + cur]
        if w.sum() > 0:
            cum = np.cumsum(w)
            i = int(np.searchsorted(cum, us[b] * cum[-1], side="right"))
            toks_b.append(i if i < V else int(np.nonzero(w)[0][-1]))
        else:
            toks_b.append(V - 1)
        out["accept_len"].append(len(path) - 1)
        out["n_out"].append(len(toks_b))
        out["out_tok"].append(toks_b + [-9] * (width - len(toks_b)))
        out["path_row"].append(path + [-9] * (width - len(path)))
        r0 += len(par)
    return {k: np.asarray(v, np.int32) for k, v in out.items()}


def counted(t):
    x = t.double().cpu().numpy()
    return np.where(np.isfinite(x) & (x > 0), x, 0.0)


def verify(eng, pars, toks, p, q, ua, us):
    for n in ("accept_len", "n_out", "out_tok", "path_row"):
        eng.st[n].fill_(-9)
    m = eng.set_rows([None if par is None else dict(tok=t, parent=par, pos=7 + depths(par)) for par, t in zip(pars, toks)])
    assert m == len(ua) <= p.shape[0]
    eng.accept_probs(p, q, torch.as_tensor(ua, dtype=torch.float32, device="cuda:0"),
                     torch.as_tensor(us, dtype=torch.float32, device="cuda:0"))
    torch.cuda.synchronize()
    return {n: eng.st[n][:len(pars)].cpu().numpy() for n in ("accept_len", "n_out", "out_tok", "path_row")}


def check(eng, pars, toks, p, q, ua, us):
    got = verify(eng, pars, toks, p, q, ua, us)
    V = eng.shape.vocab
    want = definition(pars, toks, counted(p[:, :V]), None if q is None else counted(q[:, :V]),
                      np.float32(ua).astype(np.float64), np.float32(us).astype(np.float64), eng.k_max + 1)
    for n in want:
        assert (got[n] == want[n]).all(), (n, got[n], want[n])
    return got


def uniforms(rng, n):
    return rng.integers(0, 1 << 24, n) / float(1 << 24)


def distributions(m, vocab, sharp, near, dtype, seed, pad=0):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    lg = torch.randn(m, vocab, generator=g, device="cuda:0") * sharp
    qg = lg * (1 - near * 0.1) + near * torch.randn(m, vocab, generator=g, device="cuda:0")
    out = []
    for x in (lg, qg):
        t = torch.full((m, vocab + pad), 3.0, device="cuda:0", dtype=dtype)      # (what lies behind the vocabulary is no token)
        t[:, :vocab] = torch.softmax(x, -1).to(dtype)
        out.append(t)
    return out


def drafted(pars, d, vocab, rng):
    """Tokens of every node, drawn from row `parent` of d."""
    toks, r0 = [], 0
    for par in pars:
        if par is None:
            toks.append(None)
            continue
        rows = d[r0 + np.maximum(par, 0), :vocab].double().cpu().numpy()
        toks.append(np.asarray([rng.choice(vocab, p=x / x.sum()) for x in rows], np.int32))
        r0 += len(par)
    return toks


SHAPES = ["chain", "fork", "wide", "any"]


def shapes(kind, n, rng):
    if kind == "chain":
        pars = [chain(int(rng.integers(0, 9))) for _ in range(n)]
    elif kind == "fork":                      # two branches of a step with two candidates
        pars = [np.asarray([-1, 0, 1, 2, int(rng.integers(0, 3)), 4, 5]) for _ in range(n)]
    elif kind == "wide":                      # many children of one node
        pars = [np.asarray([-1] + [0] * 7 + [1, 8, 8, 8]) for _ in range(n)]
    else:
        pars = [random_tree(int(rng.integers(1, 18)), rng) for _ in range(n)]
    pars[n // 2] = None                       # a finished sequence
    return pars


@pytest.mark.parametrize("kind", SHAPES)
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("vocab,dtype,pad,sharp", [(11, torch.float32, 0, 1.0), (3000, torch.float32, 5, 4.0), (4096, torch.bfloat16, 0, 4.0),
                                                   (10007, torch.bfloat16, 1, 6.0), (20000, torch.float32, 0, 7.0)])
def test_acceptance(kind, drawn, vocab, dtype, pad, sharp):
    rng = np.random.default_rng(vocab)
    n = 24
    for c_max in (1, 2):                      # (whatever the number of launches that sum)
        eng = engine(1, 1, 64, [8] * n, 18 if c_max == 1 else 17, vocab=vocab, c_max=c_max, max_rows=n * 18)
        taken = 0
        for trial in range(2):
            pars = shapes(kind, n, rng)
            m = sum(len(x) for x in pars if x is not None)
            p, q = distributions(m, vocab, sharp, 0.7, dtype, trial, pad)
            toks = drafted(pars, q if drawn else p, vocab, rng)
            got = check(eng, pars, toks, p, q if drawn else None, uniforms(rng, m), uniforms(rng, n))
            taken += int(got["accept_len"].sum())
        assert taken > 0
        eng.close()


def test_the_ends_of_the_random_numbers():
    """0 accepts whatever has a probability and samples the first token that has one; 1 - 2^-24 the last such token."""
    rng, vocab, n = np.random.default_rng(1), 5000, 6
    eng = engine(1, 1, 64, [8] * n, 9, vocab=vocab)
    pars = [chain(4)] * n
    p, q = distributions(5 * n, vocab, 3.0, 0.7, torch.float32, 3)
    p[:, :40] = 0
    p[:, 4800:] = 0
    toks = drafted(pars, p, vocab, rng)
    got = check(eng, pars, toks, p, q, np.zeros(5 * n), np.zeros(n))
    assert (got["accept_len"] == 4).all() and (got["out_tok"][:, 4] == 40).all()
    high = np.full(5 * n, 1.0 - 2.0 ** -24)
    got = check(eng, pars, toks, p, q, high, high[:n])
    check(eng, pars, toks, p, None, high, np.zeros(n))
    got = check(eng, pars, toks, p, None, np.zeros(5 * n), high[:n])
    assert (got["out_tok"][:, 4] < 4800).all()
    eng.close()


def test_a_draft_model_that_is_the_target():
    """q = p: everything is accepted, whatever the numbers; where nothing can be left, the sample is the target's."""
    rng, vocab, n = np.random.default_rng(2), 4099, 8
    eng = engine(1, 1, 64, [8] * n, 9, vocab=vocab)
    pars = [chain(8)] * n
    p, _ = distributions(9 * n, vocab, 3.0, 0.7, torch.float32, 4)
    toks = drafted(pars, p, vocab, rng)
    got = check(eng, pars, toks, p, p, np.full(9 * n, 1.0 - 2.0 ** -24), uniforms(rng, n))
    assert (got["accept_len"] == 8).all()
    q = (p * 1.5).contiguous()                # (no distribution, but then nothing is left behind a rejection)
    got = check(eng, pars, toks, p, q, np.full(9 * n, 0.9), uniforms(rng, n))
    assert (got["accept_len"] == 0).all()
    eng.close()


def test_probabilities_that_are_none():
    """NaN, infinities and negative values count as 0, in p and in q; empty rows; drafted ids outside the vocabulary."""
    rng, vocab, n = np.random.default_rng(3), 5001, 8
    nan, inf = float("nan"), float("inf")
    for c_max in (1, 2):
        eng = engine(1, 1, 64, [8] * n, 9, vocab=vocab, c_max=c_max)
        pars = [random_tree(7, rng) for _ in range(n)]
        m = 7 * n
        p, q = distributions(m, vocab, 3.0, 0.7, torch.float32, 5)
        toks = drafted(pars, q, vocab, rng)
        for t, bad in ((p, (nan, inf, -inf, -0.5)), (q, (inf, nan, -2.0, -inf))):
            for i, x in enumerate(bad):
                t[:, 100 * i:100 * i + 50] = x
        toks[1][2], toks[2][1], toks[3][3] = -1, vocab, 2 ** 31 - 1
        p[7 * 4:7 * 5] = 0                    # sequence 4: nothing anywhere
        p[7 * 5:7 * 6] = nan
        got = check(eng, pars, toks, p, q, uniforms(rng, m), uniforms(rng, n))
        assert got["out_tok"][4, 0] == vocab - 1 and got["out_tok"][5, 0] == vocab - 1
        check(eng, pars, toks, p, None, uniforms(rng, m), uniforms(rng, n))
        eng.close()


def test_a_very_large_vocabulary():
    """More units and slices than a workgroup keeps or a wavefront has lanes for."""
    vocab, m = 5000003, 6
    rng = np.random.default_rng(6)
    eng = engine(1, 1, 64, [8, 8], 3, vocab=vocab)
    p, q = distributions(m, vocab, 5.0, 0.5, torch.float32, 4)
    out = torch.empty(m, vocab, device="cuda:0")
    x = torch.randn(m, vocab, device="cuda:0") * 3
    eng.probs(x, out, 0.9)
    e = torch.exp((x.double() - x.double().amax(-1, keepdim=True)) / 0.9)
    # (as in _check_probs, with sums of 5000 units, 78 of them one after the other per lane)
    want = e / e.sum(-1, keepdim=True)
    assert ((out.double() - want).abs() <= want * 2.0 ** -24 * 300 + 2.0 ** -125).all()
    pars = [chain(2), np.asarray([-1, 0, 0])]
    toks = drafted(pars, q, vocab, rng)
    for _ in range(3):
        check(eng, pars, toks, p, q, uniforms(rng, m), uniforms(rng, 2))
        check(eng, pars, toks, p, None, uniforms(rng, m), uniforms(rng, 2))
    eng.close()


def test_rows_far_apart():
    """Rows whose places pass 32 bits, in elements and in bytes."""
    vocab, m, far = 1003, 3, (1 << 30) + 24
    rng = np.random.default_rng(5)
    stores = [torch.empty(far * (m - 1) + vocab, device="cuda:0", dtype=torch.bfloat16) for _ in range(2)]
    p, q = [t.as_strided((m, vocab), (far, 1)) for t in stores]
    near = distributions(m, vocab, 4.0, 0.7, torch.bfloat16, 3)
    x = torch.randn(m, vocab, device="cuda:0").to(torch.bfloat16)
    eng = engine(1, 1, 64, [8], m, vocab=vocab)
    p.copy_(x)
    eng.probs(p, q, 0.7)
    want = torch.empty_like(x)
    eng.probs(x, want, 0.7)
    assert torch.equal(q, want)
    p.copy_(near[0])
    q.copy_(near[1])
    pars = [chain(m - 1)]
    toks = drafted(pars, near[1], vocab, rng)
    for _ in range(4):
        ua, us = uniforms(rng, m), uniforms(rng, 1)
        check(eng, pars, toks, p, q, ua, us)
        check(eng, pars, toks, p, None, ua, us)
    check(eng, pars, toks, p, q, np.zeros(m), uniforms(rng, 1))      # (all accepted: the last row)
    eng.close()


def test_children_with_the_same_token():
    rng, vocab, n = np.random.default_rng(4), 300, 16
    eng = engine(1, 1, 64, [8] * n, 9, vocab=vocab, c_max=2)
    pars = [np.asarray([-1, 0, 0, 0, 1, 2])] * n
    m = 6 * n
    p, q = distributions(m, vocab, 2.0, 0.7, torch.float32, 6)
    toks = [np.asarray([0, 5, 5, 5, 7, 7], np.int32)] * n
    for d in (q, None):
        for _ in range(3):
            check(eng, pars, toks, p, d, uniforms(rng, m), uniforms(rng, n))
    eng.close()


@pytest.mark.parametrize("vocab,batch", [(152064, 1), (151936, 5)])
def test_full_vocabulary(vocab, batch):
    rng = np.random.default_rng(vocab)
    eng = engine(1, 1, 64, [8] * batch, 17, vocab=vocab, c_max=2)
    pars = [np.asarray([-1, 0, 1, 2, 0, 4, 5])] * batch
    m = 7 * batch
    for seed in range(3):
        p, q = distributions(m, vocab, 5.0, 0.7, torch.float32, seed)
        toks = drafted(pars, q, vocab, rng)
        check(eng, pars, toks, p, q, uniforms(rng, m), uniforms(rng, batch))
        check(eng, pars, toks, p, None, uniforms(rng, m), uniforms(rng, batch))
    eng.close()


@pytest.mark.parametrize("kind", ["chain", "fork"])
def test_what_is_emitted_is_distributed_as_the_target(kind):
    """The first token of 40 x 512 sequences with one target distribution, drafted from another: chi-square over 9 tokens has 8
    degrees of freedom, and 37 is exceeded by chance once in 80000 times."""
    rng, vocab, n = np.random.default_rng(5), 9, 512
    eng = engine(1, 1, 64, [8] * n, 5, vocab=vocab, c_max=2)
    par = chain(1) if kind == "chain" else np.asarray([-1, 0, 0])
    target, draft = rng.dirichlet(np.ones(vocab)), rng.dirichlet(np.ones(vocab))
    m = len(par) * n
    p = torch.as_tensor(np.tile(target, (m, 1)), dtype=torch.float32, device="cuda:0")
    q = torch.as_tensor(np.tile(draft, (m, 1)), dtype=torch.float32, device="cuda:0")
    counts, taken = np.zeros(vocab), 0
    for _ in range(40):
        toks = list(rng.choice(vocab, size=(n, len(par)), p=draft).astype(np.int32))
        got = verify(eng, [par] * n, toks, p, q, uniforms(rng, m), uniforms(rng, n))
        counts += np.bincount(got["out_tok"][:, 0], minlength=vocab)
        taken += int((got["accept_len"] > 0).sum())
    want = target * 40 * n
    assert ((counts - want) ** 2 / want).sum() < 37.0
    assert 0.2 < taken / (40 * n) < 0.98
    eng.close()


def test_streams_and_graphs():
    """On a stream of its own, and recorded: every replay verifies what it finds in the buffers."""
    rng, vocab, n = np.random.default_rng(6), 20000, 12
    eng = engine(1, 1, 64, [8] * n, 9, vocab=vocab, c_max=2)
    pars = [np.asarray([-1, 0, 1, 0, 3])] * n
    m = 5 * n
    sets, names = [], ("accept_len", "n_out", "out_tok", "path_row")
    for seed in range(3):
        lg = torch.randn(m, vocab, generator=torch.Generator(device="cuda:0").manual_seed(seed), device="cuda:0") * 5
        q = distributions(m, vocab, 5.0, 0.7, torch.float32, seed)[1]
        sets.append((lg, q, torch.as_tensor(uniforms(rng, m), dtype=torch.float32, device="cuda:0"),
                     torch.as_tensor(uniforms(rng, n), dtype=torch.float32, device="cuda:0")))
    toks = drafted(pars, sets[0][1], vocab, rng)
    eng.set_rows([dict(tok=t, parent=par, pos=7 + depths(par)) for par, t in zip(pars, toks)])
    bufs, p = [t.clone() for t in sets[0]], torch.zeros(m, vocab, device="cuda:0")

    def call():
        eng.probs(bufs[0], p, 0.9)
        eng.accept_probs(p, bufs[1], bufs[2], bufs[3])

    def result(i):
        for b, t in zip(bufs, sets[i]):
            b.copy_(t)
        for x in names:
            eng.st[x].fill_(-9)

    eager = []
    for i in range(3):
        result(i)
        call()
        eager.append({x: eng.st[x].clone() for x in names})
    side = torch.cuda.Stream()
    result(1)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert all(torch.equal(eng.st[x], eager[1][x]) for x in names)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in (2, 0, 1, 0):
        result(i)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(eng.st[x], eager[i][x]) for x in names), i
        call()
    eng.close()


def test_binding_refuses_tensors():
    eng = engine(1, 1, 64, [8], 3, vocab=50)
    eng.set_rows([dict(tok=np.zeros(3, np.int32), parent=chain(2), pos=7 + np.arange(3))])
    f = lambda *s: torch.zeros(*s, device="cuda:0")
    with pytest.raises(ValueError):
        eng.probs(f(3, 49), f(3, 50))
    with pytest.raises(ValueError):
        eng.probs(f(3, 50), f(2, 50))
    with pytest.raises(ValueError):
        eng.probs(f(3, 50).half(), f(3, 50))
    with pytest.raises(ValueError):
        eng.probs(f(3, 100)[:, ::2], f(3, 50))
    with pytest.raises(ValueError):
        eng.accept_probs(f(3, 50), f(3, 50).bfloat16(), f(3), f(1))
    with pytest.raises(ValueError):
        eng.accept_probs(f(3, 50), None, f(3).double(), f(1))
    host = lambda *s: torch.zeros(*s)
    for call in (lambda: eng.probs(host(3, 50), f(3, 50)), lambda: eng.probs(f(3, 50), host(3, 50)),
                 lambda: eng.accept_probs(host(3, 50), None, f(3), f(1)), lambda: eng.accept_probs(f(3, 50), host(3, 50), f(3), f(1)),
                 lambda: eng.accept_probs(f(3, 50), None, host(3), f(1)), lambda: eng.accept_probs(f(3, 50), None, f(3), host(1))):
        with pytest.raises(ValueError, match="cuda"):        # memory that the device does not have
            call()
    eng.close()


# ---------------------------------------------------------------- a sampled step

@pytest.mark.parametrize("temp", [0.25, 0.02])
def test_sampled_decoding_with_windows_equals_hs_accept_with_its_random_numbers(temp):
    """draft -> verify (with windows) -> probs -> accept_probs -> commit, step by step, next to an engine that runs draft -> verify ->
    accept -> commit: fed with the numbers of hs_accept's generator, the two emit the same tokens.  (The toy model's logits have a standard deviation of 0.32: at a
    temperature of 0.25 a drafted token out of 4096 has a probability of about 1 %, at 0.02 the largest has nearly all.)"""
    from hs_inputs import CONFIG_SHAPES, config_seed, history_with_context, make_prompts, make_weights, mutate, rope_table
    from paper_2508_18588_amd import HS_ACCEPT_REJECTION, hs_debug_philox
    from paper_2508_18588_amd.runtime import Engine, Policy
    shape, seed, n = CONFIG_SHAPES[1], 77, 4
    w, rope = make_weights(shape, config_seed(1)), rope_table(512, shape.head_dim)
    engs = [Engine(shape, w, rope, max_batch=n, k_max=6, c_max=2, max_len=160, shuffle_pages_seed=5) for _ in range(2)]
    prompts = list(make_prompts(n, 40, shape.vocab, seed=6))
    pol = Policy(window=8, m_min=3, k_fixed=6, k_max=6)
    for e in engs:
        e.set_window([24, 0], 4)
        e.load_sequences(prompts, [50, 40, 1, 50], seq_ids=[5, 1 << 33, 7, 8])

    def start(e, hists):
        e.load_sequences(prompts, [50, 40, 1, 50], seq_ids=[5, 1 << 33, 7, 8])
        e.set_history(hists)
        e.prefill(prompts)

    def finish(e, step):
        steps = 0
        while int(e.budget_left.max()) > 0:
            step(e)
            steps += 1
            assert steps < 120
        assert e.poll_error() == 0
        return e.tokens[:n].cpu().numpy().copy(), steps

    none = [[np.zeros(0, np.int32)] * 2 for _ in prompts]
    start(engs[0], none)
    first, _ = finish(engs[0], lambda e: e.step(pol, HS_ACCEPT_REJECTION, temp, seed))
    rng = np.random.default_rng(4)
    hists = [[history_with_context(p, mutate(t[40:90], 0.15, 0.0, shape.vocab, rng), 8) for _ in range(2)] for p, t in zip(prompts, first)]
    start(engs[0], hists)
    want, steps0 = finish(engs[0], lambda e: e.step(pol, HS_ACCEPT_REJECTION, temp, seed))

    def philox(e):
        """u of every node (its position, its place among its siblings) and of every sequence's last token."""
        ro, par, pos = (e.st[x].cpu().numpy() for x in ("row_off", "parent", "pos"))
        sid = e.seq_id.cpu().numpy().astype(np.uint64)
        ctr = []
        for b in range(n):
            for i in range(ro[b], ro[b + 1]):
                kind = int((par[ro[b]:i] == par[i]).sum())
                ctr.append((pos[i], kind, sid[b] & 0xFFFFFFFF, sid[b] >> np.uint64(32)))
        return ctr, ro, pos, sid

    def words(ctr):
        c = torch.as_tensor(np.asarray(ctr, np.uint64).astype(np.uint32).view(np.int32), device="cuda:0").contiguous()
        out = torch.zeros_like(c)
        hs_debug_philox(c.data_ptr(), seed, out.data_ptr(), len(ctr), torch.cuda.current_stream().cuda_stream)
        return ((out[:, 0].cpu().numpy().view(np.uint32) >> 8) / float(1 << 24)).astype(np.float32)

    p = torch.zeros(engs[1].max_rows, shape.vocab, device="cuda:0")

    def sampled(e):
        e.draft(pol)
        e.verify()
        e.probs(e.logits, p, temp, live=True)
        ctr, ro, pos, sid = philox(e)
        ua = torch.as_tensor(words(ctr) if ctr else np.zeros(1, np.float32), device="cuda:0")
        # the last token's number belongs to the position behind the node where the walk ends: found by a first call
        us = torch.zeros(n, device="cuda:0")
        e.accept_probs(p, None, ua, us)
        path, a = e.st["path_row"].cpu().numpy(), e.st["accept_len"].cpu().numpy()
        last = [(pos[ro[b] + path[b, a[b]]] + 1 if ro[b + 1] > ro[b] else 0, 7, sid[b] & 0xFFFFFFFF, sid[b] >> np.uint64(32)) for b in range(n)]
        e.accept_probs(p, None, ua, torch.as_tensor(words(last), device="cuda:0"))
        e.commit(pol)

    start(engs[1], hists)
    got, steps1 = finish(engs[1], sampled)
    assert (got == want).all() and steps0 == steps1
    assert temp > 0.1 or steps1 < 50
    for e in engs:
        e.close()
