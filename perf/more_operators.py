"""What the speed and the results of the operators are measured on that let the responses to one prompt share its cache: attention
that reads a shared prefix once for all of them, the pages' own traffic (free, fork, reserve, compact), and the log probabilities,
entropies and best alternatives of tokens that a trainer asks for afterwards.

Where `own` is false a pass computes the plain form with elementary torch operations; where it is true it calls the framework's
entry points.  `exact` evaluates the definitions in 64 bits, sequence by sequence."""
import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

# query heads, KV heads, head size, layers: the benchmark configurations' attention shapes
HEADS = {"toy": (4, 4, 64, 2), "1.5b": (12, 2, 128, 28), "7b": (28, 4, 128, 28), "14b": (40, 8, 128, 48)}
VOCAB = 152064      # of the 7B and 14B shapes; 151936 is the 1.5B shape's, 4096 the toy's


def listed():
    return [
        # the smallest call: four responses to one short prompt, a token each -- launches and latency
        dict(name="shared toy 1x4", op="shared", heads="toy", groups=1, members=4, plo=256, phi=256, slo=20, shi=64, rows="one", idle=0.0),
        # the end of a rollout: the longest responses of one prompt are left
        dict(name="shared 1.5b 1x7", op="shared", heads="1.5b", groups=1, members=7, plo=700, phi=700, slo=900, shi=1900, rows="one", idle=0.0),
        # plain decoding: 8 prompts of 2k to 6k tokens with up to 16 responses each, some of which have ended
        dict(name="shared 7b 8x16", op="shared", heads="7b", groups=8, members=16, plo=2048, phi=6144, slo=16, shi=4096, rows="one", idle=0.1),
        # a large batch early in the rollout, drafts of 2 to 32 tokens for three quarters of the sequences
        dict(name="shared 7b 16x16 drafts", op="shared", heads="7b", groups=16, members=16, plo=1500, phi=4500, slo=1, shi=2048, rows="aimd", idle=0.0),
        # two-branch trees of 17 nodes behind one document of 8000 tokens: many rows on the same keys
        dict(name="shared 14b 1x64 tree", op="shared", heads="14b", groups=1, members=64, plo=8000, phi=8000, slo=100, shi=400, rows="tree", idle=0.0),
        # log probabilities, entropies and 20 alternatives at all nodes of 64 trees over the full vocabulary
        dict(name="logprobs 1088 rows top 20", op="logprobs", rows=1088, vocab=VOCAB, src="f32", temperature=1.0, sharp=3.0, top=20, masked=0.0, ask="all"),
        # a few rows of 16-bit logits of which most tokens are excluded
        dict(name="logprobs 7 rows bf16 top 5", op="logprobs", rows=7, vocab=151936, src="bf16", temperature=0.7, sharp=3.0, top=5, masked=0.6, ask="all"),
        # the tokens that 64 sequences have just emitted, up to 17 each, without alternatives
        dict(name="logprobs emitted B64", op="logprobs", rows=64 * 17, vocab=VOCAB, src="f32", temperature=1.0, sharp=3.0, top=0, masked=0.0, ask="emitted"),
        # the smallest turnover of pages: three new responses to a short prompt
        dict(name="turnover toy 1x4", op="turnover", heads="toy", layers=2, groups=1, members=4, plo=100, phi=100, extra=5),
        # 120 places taken by new responses to 8 prompts, all layers of the model
        dict(name="turnover 7b 8x16", op="turnover", heads="7b", layers=28, groups=8, members=16, plo=2048, phi=6144, extra=17),
        # a small cache of which half is free
        dict(name="compact toy", op="compact", heads="toy", layers=2, batch=8, lo=40, hi=250, share=0.5),
        # giving back the upper half of a cache of 2 GB and more after the short responses have ended
        dict(name="compact 7b", op="compact", heads="7b", layers=28, batch=48, lo=256, hi=1500, share=0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["shared"] * 4 + ["logprobs"] * 3 + ["turnover", "compact"])
    if op == "logprobs":
        return dict(op=op, rows=_log(rng, 1, 1088), vocab=rng.choice([4096, 16448, 151936, VOCAB, rng.randint(1, 50000)]),
                    src=rng.choice(["f32", "f32", "bf16"]), temperature=round(rng.uniform(0.3, 1.5), 2), sharp=round(rng.uniform(1.0, 5.0), 2),
                    top=rng.choice([0, 1, 5, 20, 32, rng.randint(0, 32)]), masked=rng.choice([0.0, 0.0, 0.5, 0.99]),
                    ask=rng.choice(["all", "some", "emitted"]))
    heads = rng.choice(["toy", "1.5b", "7b", "14b", "any", "any"])
    if heads == "any":
        hkv = rng.choice([1, 2, 3, 4, 8])
        heads = "%d/%d/%d" % (hkv * rng.randint(1, 8), hkv, rng.choice([64, 128]))
    hkv, hd = _heads({"heads": heads})[1:3]
    token = 4 * hkv * hd
    if op == "compact":
        layers, hi = rng.randint(1, 28), _log(rng, 16, 4000)
        batch = max(1, min(_log(rng, 1, 256), 2000000000 // (layers * token * 2 * hi)))
        return dict(op=op, heads=heads, layers=layers, batch=batch, lo=rng.randint(1, hi), hi=hi, share=round(rng.uniform(0.1, 0.9), 2))
    members, phi = _log(rng, 1, 64), _log(rng, 1, 8000)
    groups = max(1, min(_log(rng, 1, 16), 256 // members))
    if op == "turnover":
        layers = rng.randint(1, 28)
        groups = max(1, min(groups, 2000000000 // (layers * token * (phi + 64 * members))))
        return dict(op=op, heads=heads, layers=layers, groups=groups, members=members, plo=rng.randint(1, phi), phi=phi, extra=_log(rng, 1, 40))
    shi = max(1, min(_log(rng, 1, 8000), 1000000000 // (groups * members * token)))
    rows = rng.choice(["one", "one", "aimd", "chain", "tree"])
    work = 4 * hd * _heads({"heads": heads})[0] * groups * members * {"one": 1, "aimd": 6, "chain": 9, "tree": 17}[rows]
    phi, shi = max(1, min(phi, 110000000000 // work)), max(1, min(shi, 50000000000 // work))
    return dict(op=op, heads=heads, groups=groups, members=members, plo=rng.randint(max(1, phi // 4), phi), phi=phi,
                slo=rng.randint(1, shi), shi=shi, rows=rows, idle=rng.choice([0.0, 0.0, 0.2]))


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda:0").manual_seed(seed & 0x7FFFFFFF)


def _heads(case):
    return HEADS.get(case["heads"]) or tuple(int(x) for x in case["heads"].split("/")) + (1,)


def _dev(a, dtype=torch.int64):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=dtype, device="cuda:0")


def _tree(kind, k, size):
    """Parents of one sequence's nodes: a chain of k tokens behind the root, or two chains that fork early."""
    par = list(range(-1, k))
    if kind == "tree" and k:
        at = min(int(size.geometric(0.76)) - 1, k)
        for _ in range(at, k):
            par.append(at)
            at = len(par) - 1
    return np.asarray(par)


def _depths(par):
    d = np.zeros(len(par), np.int64)
    for i in range(1, len(par)):
        d[i] = d[par[i]] + 1
    return d


def _groups(case, size):
    """Sequences of each group and its prompt's length.  (All of them full where every response is still there.)"""
    sizes = [case["members"]] + [int(size.integers((case["members"] + 1) // 2, case["members"] + 1)) for _ in range(case["groups"] - 1)]
    return sizes, [int(size.integers(case["plo"], case["phi"] + 1)) for _ in sizes]


def _layout(case):
    """What the seed does not change of a shared case: prompts, own tokens, rows, and how many pages there are."""
    size = np.random.default_rng(7)
    hq, hkv, hd, _ = _heads(case)
    sizes, prompts = _groups(case, size)
    most_k = min(32 if case["rows"] == "aimd" else 8, 256 * hkv // hq - 1)
    two = 2 if case["rows"] == "tree" else 1
    most_k = min(most_k, (256 * hkv // hq - 1) // two)
    lens, pars, group = [], [], []
    for g, (n, p) in enumerate(zip(sizes, prompts)):
        for i in range(n):
            # committed tokens: the prompt, the response's own ones, the newest of which is not in the cache yet
            lens.append(p + int(size.integers(case["slo"], case["shi"] + 1)))
            if case["rows"] == "aimd":
                k = int(min(most_k, 2 * size.geometric(0.3))) if size.random() < 0.75 else 0
            else:
                k = 0 if case["rows"] == "one" else most_k
            gone = size.random() < case["idle"] and i > 0
            pars.append(np.zeros(0, np.int64) if gone else _tree(case["rows"], k, size))
            group.append(g)
    lens = np.asarray(lens)
    shared = [p // 16 for p in prompts]                    # pages that a fork shares: the prompt's full ones
    nodes = 1 + two * most_k
    own_pages = [(int(n) + nodes + 15) // 16 - shared[g] for n, g in zip(lens, group)]
    return SimpleNamespace(sizes=sizes, lens=lens, pars=pars, deps=[_depths(p) for p in pars], group=np.asarray(group), shared=shared,
                           own_pages=own_pages, pages=sum(shared) + sum(own_pages), m=sum(len(p) for p in pars), k=most_k, two=two,
                           width=max(shared[g] + n for g, n in zip(group, own_pages)))


def _table(lay, seed):
    ids = np.arange(lay.pages, dtype=np.int32)
    np.random.default_rng(seed & 0xFFFF).shuffle(ids)
    table, o = np.full((len(lay.lens), lay.width), -1, np.int32), 0
    at = []
    for n in lay.shared:
        at.append(ids[o:o + n])
        o += n
    for b, (g, n) in enumerate(zip(lay.group, lay.own_pages)):
        table[b, :len(at[g])] = at[g]
        table[b, len(at[g]):len(at[g]) + n] = ids[o:o + n]
        o += n
    return table


def _shared_inputs(case, seed):
    hq, hkv, hd, _ = _heads(case)
    lay = _layout(case)
    g = _gen(seed * 7 + 1)
    kc = torch.randn(lay.pages, hkv, 16, hd, generator=g, device="cuda:0", dtype=torch.bfloat16)
    vc = torch.randn(lay.pages, hkv, hd, 16, generator=g, device="cuda:0", dtype=torch.bfloat16)
    q = torch.randn(lay.m, hq * hd, generator=g, device="cuda:0", dtype=torch.bfloat16).mul_(1.5)
    return SimpleNamespace(op="shared", lay=lay, kc=kc, vc=vc, q=q, table=_table(lay, seed))


def _engine(hq, hkv, hd, vocab, layers=1, **kw):
    """The context of an engine whose projections are not used here: a small width."""
    from paper_2508_18588_amd.runtime import Engine
    d, f = 64, 64
    sh = SimpleNamespace(d_model=d, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, d_ffn=f, vocab=vocab, rms_eps=1e-6)
    mat = lambda r, c: torch.zeros(r, c, device="cuda:0", dtype=torch.bfloat16)
    head, ones = mat(vocab, d), torch.ones(d, device="cuda:0")
    w = {"embed": head, "lm_head": head, "norm_f": ones, "wqkv": [mat((hq + 2 * hkv) * hd, d)] * layers, "wo": [mat(d, hq * hd)] * layers,
         "wgate": [mat(f, d)] * layers, "wup": [mat(f, d)] * layers, "wdown": [mat(d, f)] * layers, "norm1": [ones] * layers,
         "norm2": [ones] * layers}
    kw.setdefault("keep_logits", False)
    return Engine(sh, w, torch.zeros(kw["max_len"] + 128, hd // 2, 2, device="cuda:0"), **kw)


def prepare(case, seed):
    return {"shared": _prepare_shared, "logprobs": _prepare_logprobs, "turnover": _prepare_turnover, "compact": _prepare_compact}[case["op"]](case, seed)


def _prepare_shared(case, seed):
    s, (hq, hkv, hd, _) = _shared_inputs(case, seed), _heads(case)
    lay, B = s.lay, len(s.lay.lens)
    off = np.concatenate([[0], np.cumsum(lay.sizes)])
    if own:
        nodes = 1 + lay.two * lay.k
        eng = _engine(hq, hkv, hd, 4096, max_batch=B, k_max=lay.k, c_max=lay.two, max_len=16 * lay.width - nodes, pages=lay.pages)
        eng.kc.copy_(s.kc.view(torch.int16).view(-1))
        eng.vc.copy_(s.vc.view(torch.int16).view(-1))
        eng.block_table.copy_(torch.from_numpy(s.table))
        eng.load_sequences([np.zeros(int(n), np.int32) for n in lay.lens], [1000] * B)
        eng.set_rows([None if len(p) == 0 else dict(tok=np.zeros(len(p), np.int32), parent=p, pos=int(n) - 1 + d)
                      for n, p, d in zip(lay.lens, lay.pars, lay.deps)])
        eng.set_shared_prefix(off, [16 * n for n in lay.shared])
        s.eng, s.out = eng, torch.zeros_like(s.q)
        s.kc = s.vc = None
        return s
    # the plain form's indices: a group's keys and rows, a sequence's own keys and rows, each padded to a rectangle
    N, start = max(1, max(len(p) for p in lay.pars)), np.concatenate([[0], np.cumsum([len(p) for p in lay.pars])])
    P, S = 16 * np.asarray(lay.shared), np.asarray([len(p) for p in lay.pars]) + lay.lens - 1 - 16 * np.asarray(lay.shared)[lay.group]
    i = np.arange(int(P.max()))[None, :]
    s.pre_live = _dev(i < P[:, None], torch.bool)
    i = np.where(i < P[:, None], i, 0)
    first = off[:-1]
    s.pre_page, s.pre_at = _dev(s.table[first[:, None], i // 16].clip(0)), _dev(i % 16)
    own_rows = [np.arange(start[a], start[b]) for a, b in zip(off[:-1], off[1:])]
    rows = np.zeros((len(own_rows), max(1, max(len(r) for r in own_rows))), np.int64)
    back = np.zeros((lay.m, 2), np.int64)
    for g, r in enumerate(own_rows):
        rows[g, :len(r)] = r
        back[r] = np.stack([np.full(len(r), g), np.arange(len(r))], 1)
    s.pre_rows, s.pre_back = _dev(rows), _dev(back)
    slot = P[lay.group][:, None] + np.arange(int(S.max()))[None, :]
    live = np.arange(int(S.max()))[None, :] < S[:, None]
    slot = np.where(live, slot, 0)
    s.page, s.at = _dev(np.take_along_axis(s.table, slot // 16, 1).clip(0)), _dev(slot % 16)
    s.slot, s.live, s.L = _dev(slot), _dev(live, torch.bool), _dev(lay.lens - 1)
    row, back = np.zeros((B, N), np.int64), np.zeros((lay.m, 2), np.int64)
    anc = np.zeros((B, N, N), bool)
    for b, p in enumerate(lay.pars):
        row[b, :len(p)] = start[b] + np.arange(len(p))
        back[start[b]:start[b + 1]] = np.stack([np.full(len(p), b), np.arange(len(p))], 1)
        for n in range(len(p)):
            if n:
                anc[b, n] = anc[b, p[n]]
            anc[b, n, n] = True
    s.row, s.back, s.anc = _dev(row), _dev(back), _dev(anc, torch.bool)
    return s


def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _logits_inputs(case, seed):
    """Logits, the rows that are asked about, and tokens that come from the rows' distributions."""
    g = _gen(seed * 7 + 1)
    rng = np.random.default_rng(seed)
    R, V = case["rows"], case["vocab"]
    s = SimpleNamespace(op="logprobs", temperature=case["temperature"], top=min(case["top"], V), ask=case["ask"])
    s.logits = torch.randn(R, V, generator=g, device="cuda:0").mul_(case["sharp"])
    if case["masked"]:
        out = torch.rand(R, V, generator=g, device="cuda:0") < case["masked"]
        out[torch.arange(R, device="cuda:0"), s.logits.argmax(-1)] = False
        s.logits.masked_fill_(out, -math.inf)
    if s.ask == "emitted":
        # sequences of up to k + 1 rows each (a chain), of which some tokens have been accepted
        s.k = 16 if R >= 17 else R - 1
        s.batch = R // (s.k + 1)
        s.n_out = 1 + np.minimum(s.k, rng.geometric(0.4, s.batch) - 1)
        s.n_out[rng.random(s.batch) < 0.05] = 0
        s.row = np.arange(s.batch)[:, None] * (s.k + 1) + np.arange(s.k + 1)[None, :]
        s.alive = np.arange(s.k + 1)[None, :] < s.n_out[:, None]
        s.row = s.row.reshape(-1)
    else:
        s.row = np.arange(R) if s.ask == "all" else rng.integers(0, R, max(1, R // 2))
        s.alive = np.ones(len(s.row), bool)
    s.alive = s.alive.reshape(-1)
    d = torch.empty(R, V, device="cuda:0").exponential_(generator=g)
    drawn = torch.softmax(s.logits / case["temperature"], -1).div_(d).argmax(-1).cpu().numpy()
    s.logits = s.logits.to(_dtype(case["src"]) if s.ask != "emitted" else torch.float32)
    s.tok = drawn[s.row].astype(np.int32)
    return s


def _prepare_logprobs(case, seed):
    s = _logits_inputs(case, seed)
    n = len(s.row)
    s.row_dev, s.tok_dev = _dev(s.row, torch.int32), _dev(s.tok, torch.int32)
    if own:
        B, k = (s.batch, s.k) if s.ask == "emitted" else (1, 0)
        s.eng = _engine(1, 1, 64, case["vocab"], max_batch=B, k_max=min(k, 16), c_max=1, max_len=64, keep_logits=s.ask == "emitted")
        f32 = lambda *shape: torch.zeros(*shape, device="cuda:0")
        s.out = dict(logprob=f32(n), entropy=f32(n))
        if s.top:
            s.out.update(top_token=torch.zeros(n, s.top, device="cuda:0", dtype=torch.int32), top_logprob=f32(n, s.top))
        if s.ask == "emitted":
            s.eng.load_sequences([np.zeros(20, np.int32)] * B, [1000] * B)
            s.eng.set_rows([dict(tok=np.zeros(k + 1, np.int32), parent=np.arange(-1, k), pos=19 + np.arange(k + 1))] * B)
            s.eng.logits.copy_(s.logits[:B * (k + 1)])
            s.eng.st["n_out"].copy_(_dev(s.n_out, torch.int32))
            s.eng.st["out_tok"].copy_(s.tok_dev.view(B, k + 1))
            s.eng.st["path_row"].copy_(_dev(np.tile(np.arange(k + 1), (B, 1)), torch.int32))
            s.logits = None
        return s
    s.row_dev, s.tok_dev, s.alive = s.row_dev.long(), s.tok_dev.long(), _dev(s.alive, torch.bool)
    return s


def _turnover_layout(case):
    size = np.random.default_rng(7)
    sizes, prompts = _groups(case, size)
    need = [(p - 1 + 15) // 16 for p in prompts]                      # pages of a prompt's cached tokens
    first = np.concatenate([[0], np.cumsum(sizes)])[:-1]
    parent = np.repeat(first, sizes)
    per = (15 + case["extra"]) // 16 + 1                              # pages of a response's partial one and its next tokens
    return SimpleNamespace(sizes=sizes, prompts=prompts, need=need, first=first, parent=parent.astype(np.int32), batch=sum(sizes),
                           pages=sum(need) + per * sum(sizes) + 8, width=max(need) + per)


def _cache_bits(pages, layers, hkv, hd, seed):
    g = _gen(seed * 7 + 1)
    bits = lambda: torch.randint(-32768, 32767, (layers, pages, hkv * 16 * hd), generator=g, device="cuda:0", dtype=torch.int16)
    return bits(), bits()


def _turnover_inputs(case, seed):
    hq, hkv, hd, _ = _heads(case)
    lay = _turnover_layout(case)
    s = SimpleNamespace(op="turnover", lay=lay, extra=case["extra"])
    s.kc, s.vc = _cache_bits(lay.pages, case["layers"], hkv, hd, seed)
    ids = np.random.default_rng(seed & 0xFFFF).permutation(lay.pages).astype(np.int32)
    s.table, s.refs, o = np.full((lay.batch, lay.width), -1, np.int32), np.zeros(lay.pages, np.int32), 0
    s.lens = np.ones(lay.batch, np.int32)
    for b, n, p in zip(lay.first, lay.need, lay.prompts):
        s.table[b, :n] = ids[o:o + n]
        s.refs[ids[o:o + n]] = 1
        s.lens[b] = p
        o += n
    # what is released first: all that a place's last response held, and what a prompt's own sequence has beyond its text
    s.frm = np.zeros(lay.batch, np.int32)
    s.frm[lay.first] = (16 * np.asarray(lay.need)).astype(np.int32)
    s.cached = s.lens - 1
    return s


def _prepare_turnover(case, seed):
    s, (hq, hkv, hd, _) = _turnover_inputs(case, seed), _heads(case)
    lay = s.lay
    s.parent, s.frm_dev = _dev(lay.parent, torch.int32), _dev(s.frm, torch.int32)
    s.to_dev = torch.full_like(s.frm_dev, 2 ** 31 - 1)
    if own:
        eng = _engine(hq, hkv, hd, 4096, layers=case["layers"], max_batch=lay.batch, k_max=0, c_max=1, max_len=16 * lay.width - 1, pages=lay.pages)
        eng.kc.copy_(s.kc.view(-1))
        eng.vc.copy_(s.vc.view(-1))
        eng.load_sequences([np.zeros(int(n), np.int32) for n in s.lens], [1000] * lay.batch)
        eng.block_table.copy_(torch.from_numpy(s.table))
        eng.page_refs.copy_(torch.from_numpy(s.refs))
        s.eng, s.kc, s.vc = eng, None, None
        return s
    s.table, s.refs, s.lens = _dev(s.table, torch.int32), _dev(s.refs, torch.int32), _dev(s.lens, torch.int32)
    s.column, s.row = torch.arange(lay.width, device="cuda:0")[None, :], torch.arange(lay.batch, device="cuda:0")
    s.who = _dev([b for b, p in enumerate(lay.parent) if b != p and (int(s.cached[p])) % 16])
    return s


def _compact_inputs(case, seed):
    hq, hkv, hd, _ = _heads(case)
    size = np.random.default_rng(7)
    lens = size.integers(case["lo"], case["hi"] + 1, case["batch"])
    need = [(int(n) + 15) // 16 for n in lens]
    pages = sum(need)
    stays = size.permutation(case["batch"]) < max(1, round(case["share"] * case["batch"]))
    s = SimpleNamespace(op="compact", pages=pages, width=max(need), batch=case["batch"])
    s.kc, s.vc = _cache_bits(pages, case["layers"], hkv, hd, seed)
    ids, o = np.random.default_rng(5).permutation(pages).astype(np.int32), 0
    s.table, s.refs = np.full((case["batch"], s.width), -1, np.int32), np.zeros(pages, np.int32)
    for b, n in enumerate(need):
        if stays[b]:
            s.table[b, :n] = ids[o:o + n]
            s.refs[ids[o:o + n]] = 1
        o += n
    return s


def _prepare_compact(case, seed):
    s, (hq, hkv, hd, _) = _compact_inputs(case, seed), _heads(case)
    s.table0, s.refs0 = _dev(s.table, torch.int32), _dev(s.refs, torch.int32)
    if own:
        eng = _engine(hq, hkv, hd, 4096, layers=case["layers"], max_batch=s.batch, k_max=0, c_max=1, max_len=16 * s.width - 1, pages=s.pages)
        eng.kc.copy_(s.kc.view(-1))
        eng.vc.copy_(s.vc.view(-1))
        eng.load_sequences([np.zeros(1, np.int32)] * s.batch, [1000] * s.batch)
        s.eng, s.kc, s.vc = eng, None, None
        return s
    s.table, s.refs = s.table0.clone(), s.refs0.clone()
    s.page = torch.arange(s.pages, device="cuda:0")
    s.moves = int((s.refs0[int((s.refs0 > 0).sum()):] > 0).sum())
    return s


# ---------------------------------------------------------------- the pass

def run(s):
    if own:
        eng = s.eng
        if s.op == "shared":
            eng.attention_shared(0, s.q, s.out)
            return s.out
        if s.op == "logprobs":
            if s.ask == "emitted":
                eng.emitted_logprobs(s.out, s.temperature)
            else:
                eng.logprobs(s.logits, s.tok_dev, s.out, s.temperature, rows=None if s.ask == "all" else s.row_dev)
            return s.out
        if s.op == "turnover":
            eng.free_pages(s.frm_dev, s.to_dev)
            eng.fork(s.parent)
            eng.reserve(s.extra)
            return {"table": eng.block_table, "refs": eng.page_refs, "len": eng.seq_len, "k": eng.kc, "v": eng.vc}
        eng.block_table.copy_(s.table0)      # (the same pages lie apart again)
        eng.page_refs.copy_(s.refs0)
        live = eng.compact()
        return {"table": eng.block_table, "refs": eng.page_refs, "live": live, "k": eng.kc, "v": eng.vc}
    return {"shared": _plain_shared, "logprobs": _plain_logprobs, "turnover": _plain_turnover, "compact": _plain_compact}[s.op](s)


def _weights(q, k, vis):
    """Weights relative to the row's largest score, and that score."""
    x = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).mul_(1.0 / math.sqrt(q.shape[-1]))
    x = x.masked_fill_(~vis, -math.inf)
    top = x.max(-1, keepdim=True).values if x.shape[-1] else x.new_full(x.shape[:-1] + (1,), -math.inf)
    return x.sub_(top.clamp(min=-1e30)).exp_(), top


def _plain_shared(s):
    hkv, hd = s.kc.shape[1], s.kc.shape[3]
    G = s.q.shape[1] // (hkv * hd)

    def part(page, at, rows, vis):
        n, m = rows.shape
        k, v = s.kc[page, :, at].float(), s.vc[page, :, :, at].float()              # [.., keys, hkv, hd]
        q = s.q[rows].float().view(n, m, hkv, G, hd).permute(0, 2, 1, 3, 4).reshape(n, hkv, m * G, hd)
        w, top = _weights(q, k, vis)
        back = lambda t: t.view(n, hkv, m, G, -1).permute(0, 2, 1, 3, 4).reshape(n, m, hkv * G, -1)
        return back(torch.matmul(w, v.permute(0, 2, 1, 3).contiguous())), back(w.sum(-1, keepdim=True)), back(top)

    B, N = s.row.shape
    old = part(s.pre_page, s.pre_at, s.pre_rows, s.pre_live[:, None, None, :])
    old = [t[s.pre_back[:, 0], s.pre_back[:, 1]] for t in old]
    node = (s.slot - s.L[:, None]).clamp(min=0, max=N - 1)
    fresh = s.slot >= s.L[:, None]
    vis = (~fresh[:, None, :] | torch.gather(s.anc, 2, node[:, None, :].expand(B, N, -1))) & s.live[:, None, :]
    vis = vis[:, None, :, None, :].expand(B, 1, N, G, vis.shape[-1]).reshape(B, 1, N * G, -1)
    new = part(s.page, s.at, s.row, vis)
    new = [t[s.back[:, 0], s.back[:, 1]] for t in new]
    top = torch.maximum(old[2], new[2])
    a, b = torch.exp(old[2] - top), torch.exp(new[2] - top)
    out = (old[0] * a + new[0] * b) / (old[1] * a + new[1] * b)
    return out.reshape(out.shape[0], -1).to(torch.bfloat16)


def _plain_logprobs(s):
    x = s.logits.float()[s.row_dev] / s.temperature
    top = x.max(-1, keepdim=True).values
    x = x - top
    w = torch.exp(x)
    total = w.sum(-1, keepdim=True)
    log_total = torch.log(total)
    lp = torch.gather(x, 1, s.tok_dev[:, None]) - log_total
    entropy = log_total - torch.where(w > 0, w * x, torch.zeros_like(w)).sum(-1, keepdim=True) / total
    zero = lambda t: torch.where(s.alive.view(-1, *([1] * (t.dim() - 1))), t, torch.zeros_like(t))
    out = {"logprob": zero(lp[:, 0]), "entropy": zero(entropy[:, 0])}
    if s.top:
        # the largest values, the lowest index first among equal ones: keys in 64 bits, no two of which are equal
        bits = s.logits.float()[s.row_dev].add(0.0).view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * 2 ** 31 - torch.arange(x.shape[1], device="cuda:0")
        at = key.topk(s.top).indices
        out["top_token"] = zero(at.to(torch.int32))
        out["top_logprob"] = zero(torch.gather(x, 1, at) - log_total)
    return out


def _plain_turnover(s):
    lay, B = s.lay, len(s.row)
    W = lay.width
    # release
    gone = (16 * s.column >= s.frm_dev[:, None]) & (s.table >= 0)
    s.refs.index_add_(0, s.table.clamp(min=0).view(-1).long(), -gone.view(-1).to(torch.int32))
    s.table.masked_fill_(gone, -1)
    # fork: full pages are shared, the partial one is copied into the lowest free pages
    par = s.parent.long()
    child = par != s.row
    cached = s.lens[par].long() - 1
    part = child & (cached % 16 != 0)
    free = torch.sort((s.refs != 0).to(torch.int8), stable=True).indices      # the free ones in front, in order
    fresh = free[(torch.cumsum(part, 0) - 1).clamp(min=0)]
    row = torch.where(s.column < (cached // 16)[:, None], s.table[par], -1)
    at = (cached // 16).clamp(max=W - 1)
    src = s.table[par, at].long()
    row = torch.where((s.column == at[:, None]) & part[:, None], fresh[:, None].to(torch.int32), row)
    s.table.copy_(torch.where(child[:, None], row, s.table))
    added = (child[:, None] & (row >= 0)).view(-1).to(torch.int32)
    s.refs.index_add_(0, row.clamp(min=0).view(-1).long(), added)
    s.lens.copy_(torch.where(child, s.lens[par], s.lens))
    src, dst = src[s.who], fresh[s.who]
    s.kc[:, dst] = s.kc[:, src]
    s.vc[:, dst] = s.vc[:, src]
    # reserve
    L = s.lens.long()[:, None] - 1
    want = (s.column >= L // 16) & (16 * s.column < L + s.extra) & (s.table < 0)
    free = torch.sort((s.refs != 0).to(torch.int8), stable=True).indices
    more = free[(torch.cumsum(want.view(-1), 0) - 1).clamp(min=0)].view(B, W).to(torch.int32)
    s.table.copy_(torch.where(want, more, s.table))
    s.refs.index_add_(0, more.view(-1).long(), want.view(-1).to(torch.int32))
    return {"table": s.table, "refs": s.refs, "len": s.lens, "k": s.kc.view(-1), "v": s.vc.view(-1)}


def _plain_compact(s):
    s.table.copy_(s.table0)      # (the same pages lie apart again)
    s.refs.copy_(s.refs0)
    used = s.refs > 0
    live = used.sum()
    high, hole = used & (s.page >= live), ~used & (s.page < live)
    src = torch.sort((~high).to(torch.int8), stable=True).indices[:s.moves]
    dst = torch.sort((~hole).to(torch.int8), stable=True).indices[:s.moves]
    s.kc[:, dst] = s.kc[:, src]
    s.vc[:, dst] = s.vc[:, src]
    to = s.page.clone()
    to[src] = dst
    s.refs[dst] = s.refs0[src]
    s.refs.masked_fill_(s.page >= live, 0)
    s.table.copy_(torch.where(s.table >= 0, to[s.table.clamp(min=0).long()].to(torch.int32), s.table))
    return {"table": s.table, "refs": s.refs, "live": live.to(torch.int32).view(1), "k": s.kc.view(-1), "v": s.vc.view(-1)}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"] == "shared":
        hq, hkv, hd, _ = _heads(case)
        lay = _layout(case)
        keys, pairs = 0, 0
        for g, n in enumerate(lay.sizes):
            if any(len(p) for p, at in zip(lay.pars, lay.group) if at == g):
                keys += 16 * lay.shared[g]
        for n, d, g in zip(lay.lens, lay.deps, lay.group):
            if len(d):
                keys += int(n) - 1 - 16 * lay.shared[g] + len(d)
                pairs += int((int(n) + d).sum())
        return {"bytes": keys * 4.0 * hkv * hd + lay.m * 4.0 * hq * hd, "flops": 4.0 * hd * hq * pairs}
    if case["op"] == "logprobs":
        s = case["rows"]
        # (an emitted step: what the sequences have accepted is known only with the seed, 2.4 tokens each at the rates used here)
        n = float(s if case["ask"] == "all" else max(1, s // 2) if case["ask"] == "some" else min(s, max(1, s // 17) * 2.4)) * case["vocab"]
        return {"bytes": n * (2.0 if case["src"] == "bf16" and case["ask"] != "emitted" else 4.0), "flops": 6.0 * n}
    hq, hkv, hd, _ = _heads(case)
    page = 2.0 * 2 * 16 * hkv * hd * case["layers"]
    if case["op"] == "turnover":
        lay = _turnover_layout(case)
        copies = sum(n - 1 for n, p in zip(lay.sizes, lay.prompts) if (p - 1) % 16)
        return {"bytes": 2 * page * copies + 8.0 * lay.batch * lay.width + 8.0 * lay.pages, "flops": 0.0}
    lens = np.random.default_rng(7).integers(case["lo"], case["hi"] + 1, case["batch"])
    pages = sum((int(n) + 15) // 16 for n in lens)
    # (a page in random order is beyond the last one to stay with the share that goes)
    return {"bytes": 2 * page * pages * case["share"] * (1 - case["share"]) + 8.0 * pages, "flops": 0.0}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    return {"shared": _exact_shared, "logprobs": _exact_logprobs, "turnover": _exact_turnover, "compact": _exact_compact}[case["op"]](case, seed)


def _exact_shared(case, seed):
    s, (hq, hkv, hd, _) = _shared_inputs(case, seed), _heads(case)
    lay, outs, r, G = s.lay, [], 0, hq // hkv
    for b, n in enumerate(lay.lens):
        nn, L = len(lay.pars[b]), int(n) - 1
        if nn == 0:
            continue
        total = L + nn
        pages = _dev(s.table[b, :(total + 15) // 16])
        k = s.kc[pages].permute(1, 0, 2, 3).reshape(hkv, -1, hd)[:, :total].double()
        v = s.vc[pages].permute(1, 0, 3, 2).reshape(hkv, -1, hd)[:, :total].double()
        vis = np.zeros((nn, total), bool)
        vis[:, :L] = True
        for i in range(nn):
            j = i
            while j >= 0:
                vis[i, L + j] = True
                j = int(lay.pars[b][j])
        vis = _dev(vis, torch.bool).repeat_interleave(G, 0)
        q = s.q[r:r + nn].double().view(nn, hkv, G, hd).permute(1, 0, 2, 3).reshape(hkv, nn * G, hd)
        x = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(hd)
        x = x.masked_fill(~vis[None], -math.inf)
        x = torch.exp(x - x.amax(-1, keepdim=True))
        out = torch.bmm(x, v) / x.sum(-1, keepdim=True)
        outs.append(out.view(hkv, nn, G, hd).permute(1, 0, 2, 3).reshape(nn, -1))
        r += nn
    return torch.cat(outs) if outs else torch.zeros(0, hq * hd, device="cuda:0", dtype=torch.float64)


def _exact_logprobs(case, seed):
    s = _logits_inputs(case, seed)
    res = {"logprob": [], "entropy": [], "top_token": [], "top_logprob": []}
    for i in range(0, len(s.row), 64):
        x = s.logits[_dev(s.row[i:i + 64])].double()
        tok, alive = _dev(s.tok[i:i + 64]), _dev(s.alive[i:i + 64], torch.bool)
        order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :s.top] if s.top else None
        lp = torch.log_softmax(x / case["temperature"], -1)
        p = lp.exp()
        res["logprob"].append(lp.gather(1, tok[:, None])[:, 0] * alive)
        res["entropy"].append(-torch.where(p > 0, p * lp, 0.0).sum(-1) * alive)
        if s.top:
            res["top_token"].append((order * alive[:, None]).to(torch.int32))
            res["top_logprob"].append(torch.where(alive[:, None], lp.gather(1, order), 0.0))
    return {n: torch.cat(t) for n, t in res.items() if t}


def _exact_turnover(case, seed):
    s = _turnover_inputs(case, seed)
    lay, table, refs, lens = s.lay, s.table, s.refs, s.lens
    free = lambda: [int(p) for p in np.nonzero(refs == 0)[0]]
    pool, o = free(), 0
    for b, p in enumerate(lay.parent):
        if b == p:
            continue
        lens[b] = lens[p]
        cached = int(lens[p]) - 1
        table[b] = -1
        table[b, :cached // 16] = table[p, :cached // 16]
        if cached % 16:
            table[b, cached // 16] = pool[o]
            at, to = int(table[p, cached // 16]), pool[o]
            s.kc[:, to], s.vc[:, to] = s.kc[:, at], s.vc[:, at]
            o += 1
        for page in table[b]:
            if page >= 0:
                refs[page] += 1
    pool, o = free(), 0
    for b in range(lay.batch):
        L = int(lens[b]) - 1
        for i in range(L // 16, lay.width):
            if 16 * i < L + case["extra"] and table[b, i] < 0:
                table[b, i] = pool[o]
                refs[pool[o]] = 1
                o += 1
    i32 = lambda a: _dev(a, torch.int32)
    return {"table": i32(table), "refs": i32(refs), "len": i32(lens), "k": s.kc.view(-1), "v": s.vc.view(-1)}


def _exact_compact(case, seed):
    s = _compact_inputs(case, seed)
    live = int((s.refs > 0).sum())
    holes = [p for p in range(live) if s.refs[p] == 0]
    high = [p for p in range(live, s.pages) if s.refs[p] > 0]
    to = np.arange(s.pages)
    for p, h in zip(high, holes):
        to[p] = h
        s.refs[h], s.refs[p] = s.refs[p], 0
    if high:
        a, b = _dev(np.asarray(high)), _dev(np.asarray(holes))
        s.kc[:, b], s.vc[:, b] = s.kc[:, a], s.vc[:, a]
    table = np.where(s.table >= 0, to[np.maximum(s.table, 0)], -1)
    i32 = lambda a: _dev(a, torch.int32)
    return {"table": i32(table), "refs": i32(s.refs), "live": i32([live]), "k": s.kc.view(-1), "v": s.vc.view(-1)}
