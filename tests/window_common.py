"""Attention with a window and sinks by its definition, in 64 bits, and engines whose cache holds given K and V."""
from types import SimpleNamespace

import numpy as np
import torch


def engine(hq, hkv, hd, lens, nodes, max_rows=None, c_max=1, vocab=4096, seed=0, layers=1, precise=False, spare=0):
    """An engine of one narrow layer (its projections are not used) with random K and V, in shuffled pages, for sequences of
    `lens` committed tokens; nodes = the most rows that a sequence of a step may have."""
    from paper_2508_18588_amd.runtime import Engine
    d = f = 64
    sh = SimpleNamespace(d_model=d, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, d_ffn=f, vocab=vocab, rms_eps=1e-6)
    mat = lambda r, c: torch.zeros(r, c, device="cuda:0", dtype=torch.bfloat16)
    head, ones = mat(vocab, d), torch.ones(d, device="cuda:0")
    w = {"embed": head, "lm_head": head, "norm_f": ones, "wqkv": [mat((hq + 2 * hkv) * hd, d)] * layers,
         "wo": [mat(d, hq * hd)] * layers, "wgate": [mat(f, d)] * layers, "wup": [mat(f, d)] * layers,
         "wdown": [mat(d, f)] * layers, "norm1": [ones] * layers, "norm2": [ones] * layers}
    k = (min(nodes, 64) - 1) // c_max
    extra = max(0, nodes - 1 - c_max * k) + spare
    eng = Engine(sh, w, torch.zeros(max(lens) + nodes + 64, hd // 2, 2, device="cuda:0"), max_batch=len(lens),
                 k_max=min(k, 32), c_max=c_max, max_len=max(lens), seq_caps=[int(n) + extra + nodes for n in lens],
                 shuffle_pages_seed=seed + 1, max_rows=max_rows, keep_logits=False, precise=precise)
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    for t in (eng.kc, eng.vc):
        x = torch.randn(t.numel(), generator=g, device="cuda:0")
        if precise:
            t.copy_(x)
        else:
            t.view(torch.bfloat16).copy_(x.to(torch.bfloat16))
    eng.load_sequences([np.zeros(int(n), np.int32) for n in lens], [1000] * len(lens))
    return eng


def chain(k):
    return np.arange(-1, k)


def random_tree(n, rng):
    return np.asarray([-1] + [int(rng.integers(0, i)) for i in range(1, n)])


def depths(par):
    d = np.zeros(len(par), np.int64)
    for i in range(1, len(par)):
        d[i] = d[par[i]] + 1
    return d


def lay_out(eng, lens, pars):
    """Rows with these parents behind the sequences' newest tokens; None: a sequence without rows."""
    rows = [None if p is None else dict(tok=np.zeros(len(p), np.int32), parent=p, pos=n - 1 + depths(p)) for n, p in zip(lens, pars)]
    return eng.set_rows(rows)


def lay_out_chunk(eng, counts):
    off = np.zeros(eng.max_batch + 1, np.int32)
    off[1:] = np.cumsum(counts)
    eng.st["row_off"].copy_(torch.from_numpy(off))
    return int(off[-1])


def gathered(eng, b, total, layer=0):
    """K and V of sequence b's first `total` slots, [hkv, total, hd] in 64 bits."""
    sh = eng.shape
    kc = eng.kc if eng.precise else eng.kc.view(torch.bfloat16)
    vc = eng.vc if eng.precise else eng.vc.view(torch.bfloat16)
    kc = kc.view(eng.n_layers, eng.n_blocks, sh.n_kv_heads, 16, sh.head_dim)[layer]
    vc = vc.view(eng.n_layers, eng.n_blocks, sh.n_kv_heads, sh.head_dim, 16)[layer]
    pages = eng.block_table[b, :(total + 15) // 16].long().clamp(0, eng.n_blocks - 1)      # (a bad entry: no matter what)
    k = kc[pages].permute(1, 0, 2, 3).reshape(sh.n_kv_heads, -1, sh.head_dim)[:, :total]
    v = vc[pages].permute(1, 0, 3, 2).reshape(sh.n_kv_heads, -1, sh.head_dim)[:, :total]
    return k.double(), v.double()


def visible(n, par, window, sinks, chunk=False):
    """[rows, slots] of one sequence of n committed tokens."""
    L, nn = n - 1, len(par)
    dep = np.arange(nn) if chunk else depths(par)
    key = np.concatenate([np.arange(L), L + dep])
    vis = np.zeros((nn, L + nn), bool)
    vis[:, :L] = True
    for i in range(nn):
        j = i
        while j >= 0:
            vis[i, L + j] = True
            j = j - 1 if chunk else int(par[j])
    pos = L + dep
    return vis & ((key[None, :] < sinks) | (key[None, :] > pos[:, None] - window))


def reference(eng, lens, pars, q, window, sinks, chunk=False, layer=0, blocked=None):
    """(output, average of |v| with the softmax's weights) of all rows in 64 bits; blocked(b) = slots that are not seen."""
    sh = eng.shape
    G, hd = sh.n_q_heads // sh.n_kv_heads, sh.head_dim
    outs, mags, r = [], [], 0
    for b, par in enumerate(pars):
        if par is None or len(par) == 0:
            continue
        nn, total = len(par), int(lens[b]) - 1 + len(par)
        vis = visible(int(lens[b]), par, window, sinks, chunk)
        if blocked is not None:
            vis[:, blocked(b)[:total]] = False
        vis = torch.as_tensor(vis, device="cuda:0")
        k, v = gathered(eng, b, total, layer)
        qq = q[r:r + nn].double().view(nn, sh.n_kv_heads, G, hd).permute(1, 0, 2, 3).reshape(sh.n_kv_heads, nn * G, hd)
        seen = vis.repeat_interleave(G, 0)[None]
        s = torch.where(seen, (qq[:, :, None, :] * k[:, None, :, :]).sum(-1) / np.sqrt(hd) if nn * G * total < 20000
                        else torch.matmul(qq, k.transpose(1, 2).contiguous()) / np.sqrt(hd), -float("inf"))
        top = s.amax(-1, keepdim=True)
        p = torch.where(seen, torch.exp(s - torch.where(torch.isinf(top), 0.0, top)), 0.0)
        den = p.sum(-1, keepdim=True)
        den = torch.where(den == 0, 1.0, den)
        v0 = torch.where(seen.any(1)[..., None], v, 0.0)       # (a value that no row sees may be anything)
        out, mag = torch.matmul(p, v0) / den, torch.matmul(p, v0.abs()) / den
        back = lambda t: t.view(sh.n_kv_heads, nn, G, hd).permute(1, 0, 2, 3).reshape(nn, -1)
        outs.append(back(out))
        mags.append(back(mag))
        r += nn
    return torch.cat(outs), torch.cat(mags)


def bound(out, mag):
    """What a row's result may be off by: every probability is rounded to bf16 (half a step, 2^-8 of it), a partition's output to
    fp16 (2^-11) and the result to bf16 (2^-8); the scores' 32-bit sums of 128 products move an exponent by less than 2e-5, the
    rest is 32-bit arithmetic: 1e-4 of the average magnitude covers it, and 1e-6 the smallest fp16 numbers."""
    return (2.0 ** -8 + 2.0 ** -11 + 1e-4) * mag + 2.0 ** -8 * out.abs() + 1e-6


def check(got, eng, lens, pars, q, window, sinks, **kw):
    out, mag = reference(eng, lens, pars, q, window, sinks, **kw)
    got = got[:out.shape[0]].double()
    assert torch.isfinite(got).all()
    over = ((got - out).abs() - bound(out, mag)).max().item()
    assert over <= 0, f"{over} beyond the bound, largest difference {(got - out).abs().max().item()}"
    return out


def queries(m, eng, seed=3, scale=1.5):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    dt = torch.float32 if eng.precise else torch.bfloat16
    return (torch.randn(m, eng.shape.n_q_heads * eng.shape.head_dim, generator=g, device="cuda:0") * scale).to(dt)
