"""What hs_set_shared_prefix, hs_attention_shared, hs_logprobs and the calls on pages refuse, before anything is launched (no GPU)."""
import ctypes as C

import pytest

import paper_2508_18588_amd as hs
from test_boundary_host import lib  # noqa: F401  (the library fixture)
from test_operators_host import A, _context, _refused, _state

INVALID = hs.HS_ERR_INVALID_ARG


def test_struct_sizes():
    assert C.sizeof(hs.hs_shared_prefix) == 32
    assert C.sizeof(hs.hs_shared_args) == 56
    assert C.sizeof(hs.hs_page_pool) == 24
    assert C.sizeof(hs.hs_logprobs_args) == 96


def _prefix(**change):
    return hs.hs_shared_prefix(**dict(dict(n_groups=2, max_members=3, max_prefix=100, group_off=A, prefix_len=A), **change))


BAD_PREFIXES = [dict(n_groups=0), dict(n_groups=-1), dict(n_groups=5), dict(max_members=0), dict(max_members=5), dict(max_prefix=-1),
                dict(group_off=None), dict(prefix_len=None)]


def test_set_shared_prefix(lib):  # noqa: F811
    ctx, desc, lim, keep = _context()
    before = hs.hs_workspace_bytes(ctx)
    hs.hs_set_shared_prefix(ctx, _prefix())
    hs.hs_set_shared_prefix(ctx, _prefix(n_groups=4, max_members=4, max_prefix=2 ** 31 - 1))
    hs.hs_set_shared_prefix(ctx, None)
    assert hs.hs_workspace_bytes(ctx) == before
    for bad in BAD_PREFIXES:
        _refused(lambda: hs.hs_set_shared_prefix(ctx, _prefix(**bad)), INVALID, "hs_set_shared_prefix")
    assert lib.hs_set_shared_prefix(None, None) == INVALID
    hs.hs_destroy(ctx)


@pytest.mark.parametrize("name", ["n_groups", "max_members", "max_prefix"])
@pytest.mark.parametrize("big", [2 ** 32 + 1, -2 ** 32 + 1, 2 ** 31])
def test_prefixes_beyond_32_bits(name, big):
    with pytest.raises(ValueError, match=name):
        _prefix(**{name: big})


@pytest.mark.parametrize("change,status,text", [
    (dict(layer=-1), INVALID, "layer"), (dict(layer=2), INVALID, "layer"),
    (dict(q=None), INVALID, "null"), (dict(out=None), INVALID, "null"),
    (dict(q=A + 8), INVALID, "aligned"), (dict(out=A + 2), INVALID, "aligned"),
    *[(dict(prefix=bad), INVALID, "groups") for bad in BAD_PREFIXES],
])
def test_attention_shared_refuses_arguments(lib, change, status, text):  # noqa: F811
    ctx, desc, lim, keep = _context()
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    cache, seq, step = _state()
    args = dict(dict(layer=0, q=A, out=A), **{k: v for k, v in change.items() if k != "prefix"})
    args["prefix"] = _prefix(**change.get("prefix", {}))
    _refused(lambda: hs.hs_attention_shared(ctx, cache, seq, step, hs.hs_shared_args(**args)), status, text)
    hs.hs_destroy(ctx)


def test_attention_shared_refuses_state(lib):  # noqa: F811
    ctx, desc, lim, keep = _context()
    cache, seq, step = _state()
    good = hs.hs_shared_args(0, _prefix(), A, A)
    _refused(lambda: hs.hs_attention_shared(ctx, cache, seq, step, good), hs.HS_ERR_CAPACITY, "workspace")
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    _refused(lambda: hs.hs_attention_shared(ctx, hs.hs_kv_cache(None, A, 8), seq, step, good), INVALID, "cache")
    _refused(lambda: hs.hs_attention_shared(ctx, hs.hs_kv_cache(A, A, 0), seq, step, good), INVALID, "cache")
    for b in (0, 5):
        bad = hs.hs_seq_state(b, *([A] * 7), None, 0, None)
        _refused(lambda: hs.hs_attention_shared(ctx, cache, bad, step, good), INVALID, "sequence state")
    for name in ("row_off", "row2seq", "pos", "anc_mask"):
        bad = _state()[2]
        setattr(bad, name, None)
        _refused(lambda: hs.hs_attention_shared(ctx, cache, seq, bad, good), INVALID, "step arrays")
    assert lib.hs_attention_shared(ctx, C.byref(cache), C.byref(seq), C.byref(step), None, None) == INVALID
    assert lib.hs_attention_shared(None, None, None, None, None, None) == INVALID
    hs.hs_destroy(ctx)


def _ask(**change):
    base = dict(logits=A, logits_stride=4096, logits_type=hs.HS_F32, rows=4, n=4, emitted=0, temperature=1.0, top=2, row=None, token=A, live=None,
                logprob=A, entropy=A, top_token=A, top_logprob=A)
    return hs.hs_logprobs_args(**dict(base, **change))


@pytest.mark.parametrize("change,text", [
    (dict(logits=None), "null logits"), (dict(logprob=None), "null output"), (dict(token=None), "null tokens"),
    (dict(top_token=None), "null alternatives"), (dict(top_logprob=None), "null alternatives"),
    (dict(logits_type=2), "type"), (dict(logits_type=-1), "type"), (dict(rows=-1), "rows"), (dict(n=-1), "n"),
    (dict(logits_stride=4095), "stride"), (dict(logits=A + 2), "misaligned"), (dict(logits=A + 1, logits_type=hs.HS_BF16), "misaligned"),
    (dict(top=-1), "top"), (dict(top=hs.HS_LOGPROBS_TOP + 1), "top"),
    (dict(temperature=0.0), "temperature"), (dict(temperature=-1.0), "temperature"), (dict(temperature=float("nan")), "temperature"),
    (dict(temperature=float("inf")), "temperature"), (dict(temperature=1e-38), "temperature"),
])
def test_logprobs_refuses_arguments(lib, change, text):  # noqa: F811
    ctx, desc, lim, keep = _context()
    _refused(lambda: hs.hs_logprobs(ctx, _ask()), hs.HS_ERR_CAPACITY, "workspace")
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    _refused(lambda: hs.hs_logprobs(ctx, _ask(**change)), INVALID, text)
    hs.hs_logprobs(ctx, _ask(n=0, token=None))      # nothing is asked: nothing is launched
    hs.hs_destroy(ctx)


def test_logprobs_of_emitted_tokens_refuses_state(lib):  # noqa: F811
    ctx, desc, lim, keep = _context()
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    cache, seq, step = _state()
    ask = _ask(emitted=1)
    _refused(lambda: hs.hs_logprobs(ctx, ask, None, step), INVALID, "sequence state")
    _refused(lambda: hs.hs_logprobs(ctx, ask, seq, None), INVALID, "step arrays")
    for name in ("row_off", "n_out", "out_tok", "path_row"):
        bad = _state()[2]
        setattr(bad, name, None)
        _refused(lambda: hs.hs_logprobs(ctx, ask, seq, bad), INVALID, "step arrays")
    hs.hs_destroy(ctx)


def test_logprobs_without_kept_logits(lib):  # noqa: F811
    """Where the LM head leaves row maxima only there are no logits to ask about."""
    from test_boundary_host import _good
    desc, w, lim, keep = _good()
    desc.vocab = 152064
    ctx = hs.hs_create(desc, w, lim)
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    cache, seq, step = _state()
    step.logits = None
    _refused(lambda: hs.hs_logprobs(ctx, _ask(emitted=1, logits=None), seq, step), INVALID, "no logits are kept")
    hs.hs_destroy(ctx)


def test_top_beyond_the_vocabulary(lib):  # noqa: F811
    from test_boundary_host import _good
    desc, w, lim, keep = _good()
    desc.vocab = 3
    ctx = hs.hs_create(desc, w, lim)
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    _refused(lambda: hs.hs_logprobs(ctx, _ask(top=4)), INVALID, "top")
    hs.hs_destroy(ctx)


def _calls(ctx, cache, seq, pool):
    return {"free": lambda: hs.hs_pages_free(ctx, cache, seq, pool, A, A), "fork": lambda: hs.hs_pages_fork(ctx, cache, seq, pool, A),
            "reserve": lambda: hs.hs_pages_reserve(ctx, cache, seq, pool, 4), "compact": lambda: hs.hs_pages_compact(ctx, cache, pool)}


def test_pages_refuse_state(lib):  # noqa: F811
    ctx, desc, lim, keep = _context()
    cache, seq, step = _state()
    pool = hs.hs_page_pool(A, A, A)
    for name, call in _calls(ctx, cache, seq, pool).items():
        _refused(call, hs.HS_ERR_CAPACITY, f"hs_pages_{name}: no workspace")
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    for bad in (hs.hs_kv_cache(None, A, 8), hs.hs_kv_cache(A, None, 8), hs.hs_kv_cache(A, A, 0), hs.hs_kv_cache(A + 8, A, 8)):
        for call in _calls(ctx, bad, seq, pool).values():
            _refused(call, INVALID, "cache")
    for call in _calls(ctx, hs.hs_kv_cache(A, A, hs.HS_PAGES_MAX + 1), seq, pool).values():
        _refused(call, hs.HS_ERR_UNSUPPORTED, "HS_PAGES_MAX")
    for bad in (hs.hs_page_pool(None, A, A), hs.hs_page_pool(A, None, A), hs.hs_page_pool(A, A, None), hs.hs_page_pool(A, A, A + 4)):
        for call in _calls(ctx, cache, seq, bad).values():
            _refused(call, INVALID, "page pool")
    other = hs.hs_page_pool(A, A + 64, A)
    none = hs.hs_seq_state(0, *([A] * 7), None, 0, None)
    for name in ("free", "fork", "reserve"):
        _refused(_calls(ctx, cache, seq, other)[name], INVALID, "pool's")
        _refused(_calls(ctx, cache, none, pool)[name], INVALID, "sequence state")
    _refused(lambda: hs.hs_pages_free(ctx, cache, seq, pool, None, A), INVALID, "positions")
    _refused(lambda: hs.hs_pages_free(ctx, cache, seq, pool, A, None), INVALID, "positions")
    _refused(lambda: hs.hs_pages_fork(ctx, cache, seq, pool, None), INVALID, "parents")
    _refused(lambda: hs.hs_pages_reserve(ctx, cache, seq, pool, -1), INVALID, "extra")
    with pytest.raises(ValueError, match="extra"):
        hs.hs_pages_reserve(ctx, cache, seq, pool, 2 ** 32 + 1)
    hs.hs_destroy(ctx)


def test_pages_scratch(lib):  # noqa: F811
    ctx, desc, lim, keep = _context()
    assert hs.hs_pages_scratch_bytes(ctx, 0) == hs.hs_pages_scratch_bytes(ctx, -1) == hs.hs_pages_scratch_bytes(ctx, hs.HS_PAGES_MAX + 1) == 0
    sizes = [hs.hs_pages_scratch_bytes(ctx, n) for n in (1, 64, 65, 4096, 4097, 100000, hs.HS_PAGES_MAX)]
    assert sizes == sorted(sizes) and 0 < sizes[0] and sizes[-1] < 10 * hs.HS_PAGES_MAX
    with pytest.raises(ValueError):
        hs.hs_pages_scratch_bytes(ctx, 2 ** 32 + 5)
    hs.hs_destroy(ctx)
