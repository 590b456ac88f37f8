"""What the speed and the results of three operators of a speculative rollout are measured on: attention over the paged
cache with a sliding window and sinks, the probabilities of a step's logits, and the verification of drafted tokens
against probabilities from given random numbers.

Where `own` is false a pass computes the plain form with elementary torch operations; where it is true it calls the
framework's entry points.  `exact` evaluates the definitions in 64 bits, sequence by sequence."""
import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

# query heads, KV heads, head size: the benchmark configurations' attention shapes
HEADS = {"toy": (4, 4, 64), "1.5b": (12, 2, 128), "7b": (28, 4, 128), "14b": (40, 8, 128)}
VOCAB = 152064      # of the 7B and 14B shapes; 151936 is the 1.5B shape's, 4096 the toy's


def listed():
    return [
        # the smallest call there is: one sequence, one token, a short window -- launches and latency
        dict(name="window toy B1", op="window", heads="toy", batch=1, lo=300, hi=300, window=64, sinks=4, rows="one"),
        # the end of a rollout: few sequences left, one token at a time
        dict(name="window decode 1.5b B7", op="window", heads="1.5b", batch=7, lo=700, hi=2600, window=512, sinks=4, rows="one"),
        # plain decoding of a full batch, contexts of 2k to 16k tokens
        dict(name="window decode 7b B128", op="window", heads="7b", batch=128, lo=2048, hi=16384, window=1024, sinks=4, rows="one"),
        # a long tail of lengths with drafts of 2 to 32 tokens for three quarters of the sequences, a wide window
        dict(name="window step 7b B256", op="window", heads="7b", batch=256, lo=768, hi=32768, window=4096, sinks=4, rows="aimd"),
        # two-branch trees of 17 nodes over 8192 tokens
        dict(name="window step 14b B64 tree", op="window", heads="14b", batch=64, lo=8192, hi=8192, window=2048, sinks=16, rows="tree"),
        # recomputing the cache of migrated rollouts: the next 512 tokens of 8 sequences
        dict(name="window chunk 7b 8x512", op="window", heads="7b", batch=8, lo=3585, hi=3585, window=1024, sinks=4, rows="chunk", chunk=512),
        # probabilities of all nodes of 64 trees over the full vocabulary
        dict(name="probs 1088 rows", op="probs", rows=1088, vocab=VOCAB, src="f32", dst="f32", temperature=1.0, sharp=3.0),
        # a few rows of a draft model whose logits are 16 bits wide
        dict(name="probs 7 rows bf16", op="probs", rows=7, vocab=151936, src="bf16", dst="bf16", temperature=0.7, sharp=3.0),
        # the smallest verification: four chains of 4 drawn tokens over a small vocabulary
        dict(name="accept toy B4", op="accept", batch=4, vocab=4096, draft="chain", k=4, drawn=True, dtype="f32", sharp=3.0),
        # two branches of 8 drawn tokens for 64 sequences at the full vocabulary
        dict(name="accept B64 tree", op="accept", batch=64, vocab=VOCAB, draft="tree", k=8, drawn=True, dtype="f32", sharp=6.0),
        # drafts from the history, which have no distribution: as long as their match, 1 to 16 tokens, a sixth of the batch
        dict(name="accept B128 history", op="accept", batch=128, vocab=VOCAB, draft="match", k=16, drawn=False, dtype="f32", sharp=8.0),
        # chains of a draft model, probabilities held in 16 bits
        dict(name="accept B33 chain bf16", op="accept", batch=33, vocab=151936, draft="chain", k=8, drawn=True, dtype="bf16", sharp=5.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["window"] * 4 + ["probs"] + ["accept"] * 3)
    if op == "window":
        heads = rng.choice(["toy", "1.5b", "7b", "14b", "any", "any"])
        if heads == "any":
            hkv = rng.choice([1, 2, 3, 4, 8])
            heads = "%d/%d/%d" % (hkv * rng.randint(1, 8), hkv, rng.choice([64, 128]))
        kv = 4 * _heads({"heads": heads})[1] * 128
        rows = rng.choice(["one", "one", "aimd", "tree", "chain", "chunk"])
        window, sinks = _log(rng, 1, 4096), rng.choice([0, 1, 4, 4, 16, rng.randint(0, 100)])
        if rows == "chunk":
            chunk = _log(rng, 1, 1024)
            batch = max(1, min(_log(rng, 1, 16), 4096 // chunk))
            hi = _log(rng, 1, 4096)
            return dict(op=op, heads=heads, batch=batch, lo=rng.randint(1, hi), hi=hi, window=min(window, 1024), sinks=sinks,
                        rows=rows, chunk=chunk)
        hi = _log(rng, 1, 16384)
        batch = max(1, min(_log(rng, 1, 256), 1000000000 // (kv * min(hi + 64, window + 200))))
        batch = max(1, min(batch, 4000000000 // (kv * hi)))
        return dict(op=op, heads=heads, batch=batch, lo=rng.randint(max(1, hi // 8), hi), hi=hi, window=window, sinks=sinks, rows=rows)
    if op == "probs":
        return dict(op=op, rows=_log(rng, 1, 1088), vocab=rng.choice([4096, 16448, 151936, VOCAB, rng.randint(1, 50000)]),
                    src=rng.choice(["f32", "f32", "bf16"]), dst=rng.choice(["f32", "bf16"]),
                    temperature=round(rng.uniform(0.3, 1.5), 2), sharp=round(rng.uniform(1.0, 5.0), 2))
    draft = rng.choice(["chain", "tree", "match"])
    return dict(op=op, batch=_log(rng, 1, 64), vocab=rng.choice([4096, 16448, 151936, VOCAB, rng.randint(100, 50000)]),
                draft=draft, k=rng.randint(1, 16) if draft != "tree" else rng.randint(1, 8), drawn=rng.random() < 0.6,
                dtype=rng.choice(["f32", "f32", "bf16"]), sharp=round(rng.uniform(3.0, 8.0), 2))


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda:0").manual_seed(seed & 0x7FFFFFFF)


def _heads(case):
    return HEADS.get(case["heads"]) or tuple(int(x) for x in case["heads"].split("/"))


def _tree(kind, k, size):
    """Parents of one sequence's nodes: a chain of k tokens behind the root, or two chains that fork early."""
    par = list(range(-1, k))
    if kind == "tree" and k:
        at = min(int(size.geometric(0.76)) - 1, k)
        for _ in range(at, k):
            par.append(at)
            at = len(par) - 1
    return par


def _trees(case, n):
    """The nodes of n sequences.  They belong to the case, like the lengths; what is in them comes from the seed."""
    size, out = np.random.default_rng(5), []
    for _ in range(n):
        kind = case["draft"] if case["op"] == "accept" else case["rows"]
        if kind == "aimd":
            k = int(min(32, 2 * size.geometric(0.3))) if size.random() < 0.75 else 0
        elif kind == "match":
            k = int(min(case["k"], 2 + size.geometric(0.45))) if size.random() < 0.17 else 0
        else:
            k = {"one": 0, "tree": 8, "chain": 8}[kind] if case["op"] == "window" else case["k"]
        if case["op"] == "window":                      # (a KV head has at most 256 query rows)
            k = min(k, 256 * _heads(case)[1] // _heads(case)[0] - 1)
        out.append(_tree(kind, k, size))
    return out


def _lengths(case):
    """Committed tokens of each sequence, the newest one among them."""
    size = np.random.default_rng(11)
    if case["rows"] == "aimd" and case["hi"] == 32768:       # a prompt of 512 and a response of median 4000
        n = 512 + np.exp(size.normal(math.log(4000.0), 0.8, case["batch"]))
        return np.clip(np.rint(n), case["lo"], case["hi"]).astype(np.int64)
    return size.integers(case["lo"], case["hi"] + 1, case["batch"])


def _layout(case):
    """Lengths, rows and pages of a window case: what the seed does not change."""
    lens = _lengths(case)
    if case["rows"] == "chunk":
        # (one sequence of the batch has its last tokens left only)
        counts = np.full(len(lens), case["chunk"])
        if len(lens) > 1:
            counts[-1] = case["chunk"] // 2 + 1
        pars = [np.arange(-1, n - 1) for n in counts]
    else:
        pars = [np.asarray(p) for p in _trees(case, len(lens))]
    deps = []
    for p in pars:
        d = np.zeros(len(p), np.int64)
        if case["rows"] == "chunk":
            d = np.arange(len(p))
        else:
            for i in range(1, len(p)):
                d[i] = d[p[i]] + 1
        deps.append(d)
    most = max(len(p) for p in pars)
    need = [(int(n) + most + 15) // 16 for n in lens]
    return SimpleNamespace(lens=lens, pars=pars, deps=deps, need=need, pages=int(sum(need)), most=most,
                           m=sum(len(p) for p in pars))


def _pages(lay, seed):
    ids = np.arange(lay.pages, dtype=np.int32)
    np.random.default_rng(seed & 0xFFFF).shuffle(ids)
    table, o = np.full((len(lay.need), max(lay.need)), -1, np.int32), 0
    for b, n in enumerate(lay.need):
        table[b, :n] = ids[o:o + n]
        o += n
    return table


def _window_inputs(case, seed):
    hq, hkv, hd = _heads(case)
    lay = _layout(case)
    g = _gen(seed * 7 + 1)
    kc = torch.randn(lay.pages, hkv, 16, hd, generator=g, device="cuda:0", dtype=torch.bfloat16)
    vc = torch.randn(lay.pages, hkv, hd, 16, generator=g, device="cuda:0", dtype=torch.bfloat16)
    q = torch.randn(lay.m, hq * hd, generator=g, device="cuda:0", dtype=torch.bfloat16).mul_(1.5)
    return SimpleNamespace(lay=lay, kc=kc, vc=vc, q=q, table=_pages(lay, seed))


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda:0")


def _engine(hq, hkv, hd, vocab, **kw):
    """The context of an engine whose projections are not used here: a small width, one layer."""
    from paper_2508_18588_amd.runtime import Engine
    d, f = 64, 64
    sh = SimpleNamespace(d_model=d, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, d_ffn=f, vocab=vocab, rms_eps=1e-6)
    mat = lambda r, c: torch.zeros(r, c, device="cuda:0", dtype=torch.bfloat16)
    head, ones = mat(vocab, d), torch.ones(d, device="cuda:0")
    w = {"embed": head, "lm_head": head, "norm_f": ones, "wqkv": [mat((hq + 2 * hkv) * hd, d)], "wo": [mat(d, hq * hd)],
         "wgate": [mat(f, d)], "wup": [mat(f, d)], "wdown": [mat(d, f)], "norm1": [ones], "norm2": [ones]}
    longest = kw["max_len"] + 64 + kw.get("room", 0)
    kw.pop("room", None)
    return Engine(sh, w, torch.zeros(longest, hd // 2, 2, device="cuda:0"), keep_logits=False, **kw)


def _rows_of(lens, pars, deps, toks=None):
    return [dict(tok=np.zeros(len(p), np.int32) if toks is None else toks[b], parent=p, pos=int(lens[b]) - 1 + deps[b])
            for b, p in enumerate(pars)]


def prepare(case, seed):
    return {"window": _prepare_window, "probs": _prepare_probs, "accept": _prepare_accept}[case["op"]](case, seed)


def _prepare_window(case, seed):
    s, (hq, hkv, hd) = _window_inputs(case, seed), _heads(case)
    lay, chunk = s.lay, case.get("chunk", 0)
    s.op, s.window, s.sinks, s.chunk = "window", case["window"], case["sinks"], chunk
    if own:
        B, k = case["batch"], 0 if chunk else (8 if case["rows"] == "tree" else max(0, lay.most - 1))
        eng = _engine(hq, hkv, hd, 4096, max_batch=B, k_max=k, c_max=2 if case["rows"] == "tree" else 1,
                      max_len=int(lay.lens.max()), seq_caps=[16 * n - (1 + k * (2 if case["rows"] == "tree" else 1)) for n in lay.need],
                      max_rows=max(lay.m, B), room=chunk)
        eng.kc.copy_(s.kc.view(torch.int16).view(-1))
        eng.vc.copy_(s.vc.view(torch.int16).view(-1))
        eng.block_table.copy_(torch.from_numpy(s.table))
        eng.load_sequences([np.zeros(int(n), np.int32) for n in lay.lens], [1000] * B)
        if chunk:
            eng.st["row_off"].copy_(_i32(np.concatenate([[0], np.cumsum([len(p) for p in lay.pars])])))
        else:
            eng.set_rows(_rows_of(lay.lens, lay.pars, lay.deps))
        s.eng, s.out = eng, torch.zeros_like(s.q)
        s.kc = s.vc = None
        return s
    # the plain form's indices: the visible keys of every sequence and the rows that see them, padded to a rectangle
    B, N = case["batch"], lay.most
    L = lay.lens - 1
    first = np.maximum(0, L + 1 - s.window)
    sink = np.minimum(s.sinks, first)
    total = L + np.asarray([len(p) for p in lay.pars])
    i = np.arange(int((sink + total - first).max()))[None, :]
    slot = np.where(i < sink[:, None], i, first[:, None] + i - sink[:, None])
    live = slot < total[:, None]
    slot = np.where(live, slot, 0)
    s.page = torch.as_tensor(np.take_along_axis(s.table, slot // 16, 1).astype(np.int64), device="cuda:0")
    s.at = torch.as_tensor(slot % 16, device="cuda:0")
    s.slot, s.live, s.L = torch.as_tensor(slot, device="cuda:0"), torch.as_tensor(live, device="cuda:0"), torch.as_tensor(L, device="cuda:0")
    pos, row, seq = np.zeros((B, N), np.int64), np.full((B, N), lay.m, np.int64), []
    for b, d in enumerate(lay.deps):
        pos[b, :len(d)] = L[b] + d
        row[b, :len(d)] = len(seq) + np.arange(len(d))
        seq += [(b, n) for n in range(len(d))]
    s.pos, s.row = torch.as_tensor(pos, device="cuda:0"), torch.as_tensor(np.minimum(row, lay.m - 1), device="cuda:0")
    s.back = torch.as_tensor(np.asarray(seq), device="cuda:0")
    if not chunk:
        anc = np.zeros((B, N, N), bool)
        for b, p in enumerate(lay.pars):
            for n in range(len(p)):
                if n:
                    anc[b, n] = anc[b, p[n]]
                anc[b, n, n] = True
        s.anc = torch.as_tensor(anc, device="cuda:0")
    return s


def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _logits(case, seed, rows, salt):
    g = _gen(seed * 7 + salt)
    return torch.randn(rows, case["vocab"], generator=g, device="cuda:0").mul_(case["sharp"])


def _softmax64(x):
    x = x.double()
    x = torch.exp(x - x.max(-1, keepdim=True).values)
    return x / x.sum(-1, keepdim=True)


def _prepare_probs(case, seed):
    s = SimpleNamespace(op="probs", logits=_logits(case, seed, case["rows"], 1).to(_dtype(case["src"])),
                        temperature=case["temperature"], dst=_dtype(case["dst"]))
    if own:
        s.eng = _engine(1, 1, 64, case["vocab"], max_batch=case["rows"], k_max=0, c_max=1, max_len=16)
        s.out = torch.zeros(case["rows"], case["vocab"], device="cuda:0", dtype=s.dst)
    return s


def _accept_inputs(case, seed):
    """Target's and draft's distributions at every node, and drafted tokens that come from the draft's distribution, or,
    where it has none, from the target's largest tokens."""
    rng, pars, V = np.random.default_rng(seed), _trees(case, case["batch"]), case["vocab"]
    m = sum(len(p) for p in pars)
    dt = _dtype(case["dtype"])
    lg = _logits(case, seed, m, 1)
    noise = _gen(seed * 7 + 2)
    s = SimpleNamespace(pars=pars, m=m, p=torch.empty(m, V, device="cuda:0", dtype=dt), q=None)
    if case["drawn"]:
        s.q = torch.empty(m, V, device="cuda:0", dtype=dt)
    par_row = np.concatenate([np.where(np.asarray(p) < 0, 0, p) for p in pars]) + \
        np.repeat(np.cumsum([0] + [len(p) for p in pars])[:-1], [len(p) for p in pars])
    par_row = torch.as_tensor(par_row, device="cuda:0")
    tok = torch.empty(m, dtype=torch.int64, device="cuda:0")
    for r in range(0, m, 64):
        s.p[r:r + 64] = _softmax64(lg[r:r + 64]).to(dt)
        if case["drawn"]:
            near = 0.95 * lg[r:r + 64] + 0.5 * torch.randn(min(64, m - r), V, generator=noise, device="cuda:0")
            s.q[r:r + 64] = _softmax64(near).to(dt)
    for r in range(0, m, 64):
        at = par_row[r:r + 64]
        d = (s.q if case["drawn"] else s.p)[at].float()
        e = torch.empty(d.shape, device="cuda:0").exponential_(generator=noise)
        tok[r:r + 64] = (d / e).argmax(-1)
    s.tok = tok.cpu().numpy().astype(np.int32)
    # (24 random bits, as such generators give them)
    s.u_accept = torch.as_tensor(rng.integers(0, 1 << 24, m) / float(1 << 24), dtype=torch.float32, device="cuda:0")
    s.u_sample = torch.as_tensor(rng.integers(0, 1 << 24, len(pars)) / float(1 << 24), dtype=torch.float32, device="cuda:0")
    return s


def _prepare_accept(case, seed):
    s = _accept_inputs(case, seed)
    s.op, B, V = "accept", case["batch"], case["vocab"]
    two = 2 if case["draft"] == "tree" else 1
    s.width = case["k"] + 1
    if own:
        eng = _engine(1, 1, 64, V, max_batch=B, k_max=case["k"], c_max=two, max_len=64)
        eng.load_sequences([np.zeros(20, np.int32)] * B, [1000] * B)
        o, toks, deps = 0, [], []
        for p in s.pars:
            toks.append(s.tok[o:o + len(p)])
            o += len(p)
            deps.append(np.zeros(len(p), np.int64))
        eng.set_rows(_rows_of([20] * B, [np.asarray(p) for p in s.pars], deps, toks))
        s.eng = eng
        return s
    # the plain form's structure: children of every node, padded
    most = max(len(p) for p in s.pars)
    kids = np.full((B, most, most), -1, np.int64)
    for b, p in enumerate(s.pars):
        for i in range(1, len(p)):
            kids[b, p[i], int((kids[b, p[i]] >= 0).sum())] = i
    s.children = max(1, int((kids >= 0).sum(-1).max()))
    s.kids = torch.as_tensor(kids[:, :, :s.children], device="cuda:0")
    s.first = torch.as_tensor(np.cumsum([0] + [len(p) for p in s.pars])[:-1], device="cuda:0")
    s.tok64 = torch.as_tensor(s.tok.astype(np.int64), device="cuda:0")
    return s


# ---------------------------------------------------------------- the pass

def run(s):
    if own:
        if s.op == "window":
            s.eng.attention_window(0, s.q, s.out, s.window, s.sinks, s.chunk)
            return s.out
        if s.op == "probs":
            s.eng.probs(s.logits, s.out, s.temperature)
            return s.out
        s.eng.accept_probs(s.p, s.q, s.u_accept, s.u_sample)
        return {n: s.eng.st[n] for n in ("accept_len", "n_out", "out_tok", "path_row")}
    return {"window": _plain_window, "probs": _plain_probs, "accept": _plain_accept}[s.op](s)


def _plain_window(s):
    hkv, hd = s.kc.shape[1], s.kc.shape[3]
    B, N = s.pos.shape
    G = s.q.shape[1] // (hkv * hd)
    k = s.kc[s.page, :, s.at].float()                               # [B, keys, hkv, hd]
    v = s.vc[s.page, :, :, s.at].float()
    q = s.q[s.row].float().view(B, N, hkv, G, hd).permute(0, 2, 1, 3, 4).reshape(B, hkv, N * G, hd)
    score = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).mul_(1.0 / math.sqrt(hd))
    # a key's position: its slot, or the depth of the draft node that lies there
    node = (s.slot - s.L[:, None]).clamp(min=0)                     # [B, keys]
    fresh = s.slot >= s.L[:, None]
    if s.chunk:
        key, seen = s.slot, torch.ones((), dtype=torch.bool, device="cuda:0")
        vis = s.slot[:, None, :] <= s.pos[:, :, None]
    else:
        node = node.clamp(max=N - 1)
        key = torch.where(fresh, torch.gather(s.pos, 1, node), s.slot)
        seen = torch.gather(s.anc, 2, node[:, None, :].expand(B, N, -1))
        vis = ~fresh[:, None, :] | seen
    vis = vis & s.live[:, None, :] & ((key[:, None, :] > s.pos[:, :, None] - s.window) | (key[:, None, :] < s.sinks))
    vis = vis[:, None, :, None, :].expand(B, 1, N, G, vis.shape[-1]).reshape(B, 1, N * G, -1)
    score = score.masked_fill_(~vis, -math.inf)
    score = torch.exp(score.sub_(score.max(-1, keepdim=True).values))
    den = score.sum(-1, keepdim=True)
    out = torch.matmul(score, v.permute(0, 2, 1, 3).contiguous()) / den
    out = out.view(B, hkv, N, G, hd).permute(0, 2, 1, 3, 4).reshape(B, N, hkv * G * hd)
    return out[s.back[:, 0], s.back[:, 1]].to(torch.bfloat16)


def _plain_probs(s):
    x = s.logits.float() / s.temperature
    x = torch.exp(x - x.max(-1, keepdim=True).values)
    return (x / x.sum(-1, keepdim=True)).to(s.dst)


def _left(s, row, rejected, toks):
    """Weights at each sequence's node after `rejected` of its children: [B, V] in 64 bits, and the sums on the way."""
    w, z = s.p[row].double(), torch.ones(len(row), dtype=torch.float64, device="cuda:0")
    q = None if s.q is None else s.q[row].double()
    for j in range(toks.shape[1]):
        if q is None:
            nxt = w.scatter(1, toks[:, j:j + 1], 0.0)
        else:
            nxt = (w - z[:, None] * q).clamp_(min=0.0)
        go = rejected > j
        w = torch.where(go[:, None], nxt, w)
        z = torch.where(go, w.sum(1), z)
    return w, z


def _plain_accept(s):
    B, dev = len(s.pars), "cuda:0"
    cur, a = torch.zeros(B, dtype=torch.int64, device=dev), torch.zeros(B, dtype=torch.int64, device=dev)
    out = torch.zeros(B, s.width, dtype=torch.int64, device=dev)
    path = torch.zeros(B, s.width, dtype=torch.int64, device=dev)
    over = torch.zeros(B, dtype=torch.bool, device=dev)
    rej = torch.zeros(B, dtype=torch.int64, device=dev)
    seq = torch.arange(B, device=dev)
    depth = s.width - 1
    for level in range(depth):
        kid = s.kids[seq, cur]                                       # [B, children]
        row, toks = s.first + cur, s.tok64[s.first[:, None] + kid.clamp(min=0)]
        nxt, n = torch.full_like(cur, -1), torch.zeros_like(cur)
        for j in range(s.children):
            if j == 0:
                w_t, z = s.p[row, toks[:, 0]].double(), torch.ones(B, dtype=torch.float64, device=dev)
            else:
                w, z = _left(s, row, torch.full_like(cur, j), toks[:, :j])
                w_t = torch.gather(w, 1, toks[:, j:j + 1])[:, 0]
            q_t = 1.0 if s.q is None else s.q[row, toks[:, j]].double()
            u = s.u_accept[s.first + kid[:, j].clamp(min=0)].double()
            there = (kid[:, j] >= 0) & (nxt < 0) & ~over
            ok = there & (u * z * q_t < w_t)
            nxt = torch.where(ok, kid[:, j], nxt)
            n = n + (there & ~ok).long()
        go = nxt >= 0
        rej = torch.where(over, rej, torch.where(go, torch.zeros_like(n), n))
        over = over | ~go
        to = torch.where(go, nxt, torch.zeros_like(nxt))
        out[:, level] = torch.where(go, s.tok64[s.first + to], out[:, level])
        path[:, level + 1] = to
        cur, a = torch.where(go, nxt, cur), a + go.long()
    kid = s.kids[seq, cur]
    row = s.first + cur
    w, z = _left(s, row, rej, s.tok64[s.first[:, None] + kid.clamp(min=0)])
    w = torch.where((w.sum(1) > 0)[:, None], w, s.p[row].double())
    cum = w.cumsum(1)
    target = s.u_sample.double() * cum[:, -1]
    pick = torch.searchsorted(cum, target[:, None], right=True)[:, 0].clamp(max=w.shape[1] - 1)
    out[seq, a] = pick
    i32 = lambda t: t.to(torch.int32)
    return {"accept_len": i32(a), "n_out": i32(a + 1), "out_tok": i32(out), "path_row": i32(path)}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"] == "window":
        hq, hkv, hd = _heads(case)
        lay = _layout(case)
        keys = pairs = 0
        for n, dep in zip(lay.lens, lay.deps):
            L = int(n) - 1
            first = max(0, L + 1 - case["window"])
            keys += min(case["sinks"], first) + L + len(dep) - first
            pos = L + dep
            lo = np.maximum(0, pos + 1 - case["window"])
            pairs += int((pos + 1 - lo + np.minimum(case["sinks"], lo)).sum())
        return {"bytes": keys * 4.0 * hkv * hd + lay.m * 4.0 * hq * hd, "flops": 4.0 * hd * hq * pairs}
    size = {"f32": 4.0, "bf16": 2.0}
    if case["op"] == "probs":
        n = float(case["rows"]) * case["vocab"]
        return {"bytes": n * (size[case["src"]] + size[case["dst"]]), "flops": 4.0 * n}
    # one row of the target's, and of the draft's where there is one, per sequence
    n = float(case["batch"]) * case["vocab"] * (2 if case["drawn"] else 1)
    return {"bytes": n * size[case["dtype"]], "flops": 2.0 * n}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    return {"window": _exact_window, "probs": _exact_probs, "accept": _exact_accept}[case["op"]](case, seed)


def _exact_window(case, seed):
    s, (hq, hkv, hd) = _window_inputs(case, seed), _heads(case)
    lay, outs, r = s.lay, [], 0
    for b, n in enumerate(lay.lens):
        nn, L = len(lay.pars[b]), int(n) - 1
        total = L + nn
        pages = torch.as_tensor(s.table[b, :(total + 15) // 16].astype(np.int64), device="cuda:0")
        k = s.kc[pages].permute(1, 0, 2, 3).reshape(hkv, -1, hd)[:, :total]
        v = s.vc[pages].permute(1, 0, 3, 2).reshape(hkv, -1, hd)[:, :total]
        pos = L + torch.as_tensor(np.asarray(lay.deps[b]), device="cuda:0")
        key = torch.cat([torch.arange(L, device="cuda:0"), pos])
        vis = torch.zeros(nn, total, dtype=torch.bool, device="cuda:0")
        vis[:, :L] = True
        if case["rows"] == "chunk":
            vis[:, L:] = torch.tril(torch.ones(nn, nn, dtype=torch.bool, device="cuda:0"))
        else:
            up = np.zeros((nn, nn), bool)
            for i in range(nn):
                j = i
                while j >= 0:
                    up[i, j] = True
                    j = int(lay.pars[b][j])
            vis[:, L:] = torch.as_tensor(up, device="cuda:0")
        vis &= (key[None, :] < case["sinks"]) | (pos[:, None] - key[None, :] < case["window"])
        used = vis.any(0).nonzero()[:, 0]                            # (all other keys weigh nothing)
        k, v, vis = k[:, used].double(), v[:, used].double(), vis[:, used]
        q = s.q[r:r + nn].double().view(nn, hkv, hq // hkv, hd)
        out = torch.empty(nn, hkv, hq // hkv, hd, device="cuda:0", dtype=torch.float64)
        for j in range(hkv):
            x = q[:, j].reshape(-1, hd) @ k[j].T.contiguous() / math.sqrt(hd)
            x = x.masked_fill(~vis.repeat_interleave(hq // hkv, 0), -math.inf)
            x = torch.exp(x - x.amax(-1, keepdim=True))
            out[:, j] = ((x @ v[j]) / x.sum(-1, keepdim=True)).view(nn, -1, hd)
        outs.append(out.reshape(nn, -1))
        r += nn
    return torch.cat(outs)


def _exact_probs(case, seed):
    x = _logits(case, seed, case["rows"], 1).to(_dtype(case["src"]))
    return torch.cat([_softmax64(x[r:r + 64].double() / case["temperature"]) for r in range(0, len(x), 64)])


def _exact_accept(case, seed):
    s = _accept_inputs(case, seed)
    width, V, r0 = case["k"] + 1, case["vocab"], 0
    res = {"accept_len": [], "n_out": [], "out_tok": [], "path_row": []}
    ua, us = s.u_accept.cpu().numpy().astype(np.float64), s.u_sample.cpu().numpy().astype(np.float64)
    line = lambda t, r: t[r].double().cpu().numpy()
    for b, par in enumerate(s.pars):
        cur, toks, path = 0, [], [0]
        while True:
            p = line(s.p, r0 + cur)
            q = None if s.q is None else line(s.q, r0 + cur)
            w, z, took = p, 1.0, None
            for c in [i for i in range(1, len(par)) if par[i] == cur]:
                t = int(s.tok[r0 + c])
                if ua[r0 + c] * z * (1.0 if q is None else q[t]) < w[t]:
                    took = c
                    break
                point = np.zeros(V)
                point[t] = w[t]
                w = np.maximum(w - (point if q is None else z * q), 0.0)
                z = w.sum()
            if took is None:
                break
            cur = took
            toks.append(int(s.tok[r0 + took]))
            path.append(took)
        if not w.sum() > 0:
            w = p
        cum = np.cumsum(w)
        toks.append(int(min(V - 1, np.searchsorted(cum, us[b] * cum[-1], side="right"))))
        res["accept_len"].append(len(path) - 1)
        res["n_out"].append(len(toks))
        res["out_tok"].append(toks + [0] * (width - len(toks)))
        res["path_row"].append(path + [0] * (width - len(path)))
        r0 += len(par)
    return {n: torch.as_tensor(np.asarray(x), dtype=torch.int32, device="cuda:0") for n, x in res.items()}
