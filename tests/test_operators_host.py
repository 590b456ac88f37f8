"""What hs_set_window, hs_attention_window, hs_probs and hs_accept_probs refuse, before anything is launched (no GPU)."""
import ctypes as C

import pytest

import paper_2508_18588_amd as hs
from test_boundary_host import _good, lib  # noqa: F401  (the library fixture)

A = 0x1000      # an address that is never touched


def _context():
    desc, w, lim, keep = _good()
    ctx = hs.hs_create(desc, w, lim)
    return ctx, desc, lim, (w, keep)


def _state():
    seq = hs.hs_seq_state(4, *([A] * 7), None, 0, None)
    return hs.hs_kv_cache(A, A, 8), seq, hs.hs_step(*([A] * 15), 0)


def _refused(call, status, text=None):
    with pytest.raises(hs.HsError) as e:
        call()
    assert e.value.status == status, e.value
    if text:
        assert text in str(e.value)


def test_struct_sizes():
    assert C.sizeof(hs.hs_window_args) == 32
    assert C.sizeof(hs.hs_probs_args) == 56
    assert C.sizeof(hs.hs_accept_probs_args) == 56


def test_set_window(lib):  # noqa: F811
    ctx, desc, lim, keep = _context()
    before = hs.hs_workspace_bytes(ctx)
    hs.hs_set_window(ctx, [16, 0], 4)
    hs.hs_set_window(ctx, [1, hs.HS_WINDOW_MAX], hs.HS_WINDOW_MAX)
    hs.hs_set_window(ctx, None)
    assert hs.hs_workspace_bytes(ctx) == before
    _refused(lambda: hs.hs_set_window(ctx, [16, -1], 4), hs.HS_ERR_INVALID_ARG, "window")
    _refused(lambda: hs.hs_set_window(ctx, [16, hs.HS_WINDOW_MAX + 1], 4), hs.HS_ERR_INVALID_ARG, "window")
    _refused(lambda: hs.hs_set_window(ctx, [16, 16], -1), hs.HS_ERR_INVALID_ARG, "sinks")
    assert lib.hs_set_window(None, None, 0) == hs.HS_ERR_INVALID_ARG
    hs.hs_destroy(ctx)


@pytest.mark.parametrize("change,status,text", [
    (dict(layer=-1), hs.HS_ERR_INVALID_ARG, "layer"),
    (dict(layer=2), hs.HS_ERR_INVALID_ARG, "layer"),
    (dict(window=0), hs.HS_ERR_INVALID_ARG, "window"),
    (dict(window=-5), hs.HS_ERR_INVALID_ARG, "window"),
    (dict(window=hs.HS_WINDOW_MAX + 1), hs.HS_ERR_INVALID_ARG, "window"),
    (dict(sinks=-1), hs.HS_ERR_INVALID_ARG, "sinks"),
    (dict(chunk=-1), hs.HS_ERR_INVALID_ARG, "chunk"),
    (dict(chunk=21), hs.HS_ERR_CAPACITY, "chunk"),
    (dict(q=None), hs.HS_ERR_INVALID_ARG, "null"),
    (dict(out=None), hs.HS_ERR_INVALID_ARG, "null"),
    (dict(q=A + 8), hs.HS_ERR_INVALID_ARG, "aligned"),
    (dict(out=A + 2), hs.HS_ERR_INVALID_ARG, "aligned"),
])
def test_attention_window_refuses_arguments(lib, change, status, text):  # noqa: F811
    ctx, desc, lim, keep = _context()
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    cache, seq, step = _state()
    args = dict(layer=0, window=8, sinks=4, chunk=0, q=A, out=A)
    args.update(change)
    _refused(lambda: hs.hs_attention_window(ctx, cache, seq, step, hs.hs_window_args(**args)), status, text)
    hs.hs_destroy(ctx)


def test_attention_window_refuses_state(lib):  # noqa: F811
    ctx, desc, lim, keep = _context()
    cache, seq, step = _state()
    good = hs.hs_window_args(0, 8, 4, 0, A, A)
    _refused(lambda: hs.hs_attention_window(ctx, cache, seq, step, good), hs.HS_ERR_CAPACITY, "workspace")
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    _refused(lambda: hs.hs_attention_window(ctx, hs.hs_kv_cache(A, None, 8), seq, step, good), hs.HS_ERR_INVALID_ARG, "cache")
    _refused(lambda: hs.hs_attention_window(ctx, cache, hs.hs_seq_state(5, *([A] * 7), None, 0, None), step, good),
             hs.HS_ERR_INVALID_ARG, "sequence")
    for missing in ("row_off", "pos", "anc_mask", "row2seq"):
        bad = hs.hs_step(*([A] * 15), 0)
        setattr(bad, missing, None)
        _refused(lambda: hs.hs_attention_window(ctx, cache, seq, bad, good), hs.HS_ERR_INVALID_ARG, "step")
    hs.hs_set_flags(ctx, hs.HS_FLAG_REFERENCE_KERNELS)
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    _refused(lambda: hs.hs_attention_window(ctx, cache, seq, step, hs.hs_window_args(0, 8, 4, 2, A, A)), hs.HS_ERR_UNSUPPORTED,
             "chunk")
    hs.hs_destroy(ctx)


@pytest.mark.parametrize("change,text", [
    (dict(logits=None), "null"), (dict(out=None), "null"), (dict(logits_type=2), "type"), (dict(out_type=-1), "type"),
    (dict(temperature=0.0), "temperature"), (dict(temperature=-1.0), "temperature"), (dict(temperature=float("nan")), "temperature"),
    (dict(rows=-1), "rows"), (dict(logits_stride=4095), "stride"), (dict(out_stride=4095), "stride"),
    (dict(logits=A + 2), "misaligned"), (dict(out=A + 1, out_type=hs.HS_BF16), "misaligned"),
    (dict(out=A, out_type=hs.HS_BF16), "in place"), (dict(out=A, out_stride=4100), "in place"),
])
def test_probs_refuses_arguments(lib, change, text):  # noqa: F811
    ctx, desc, lim, keep = _context()
    args = dict(logits=A, out=2 * A, logits_stride=4096, out_stride=4096, logits_type=hs.HS_F32, out_type=hs.HS_F32, rows=3,
                temperature=1.0, live_rows=None)
    _refused(lambda: hs.hs_probs(ctx, hs.hs_probs_args(**args)), hs.HS_ERR_CAPACITY, "workspace")
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    hs.hs_probs(ctx, hs.hs_probs_args(**dict(args, rows=0)))          # nothing to do, nothing launched
    args.update(change)
    _refused(lambda: hs.hs_probs(ctx, hs.hs_probs_args(**args)), hs.HS_ERR_INVALID_ARG, text)
    hs.hs_destroy(ctx)


@pytest.mark.parametrize("change,text", [
    (dict(p=None), "null"), (dict(u_accept=None), "null"), (dict(u_sample=None), "null"), (dict(type=2), "type"),
    (dict(p_stride=4095), "stride"), (dict(q_stride=4095), "stride"), (dict(p_stride=-4096), "stride"), (dict(p=A + 2), "misaligned"),
    (dict(q=A + 1, type=hs.HS_BF16), "misaligned"),
])
def test_accept_probs_refuses_arguments(lib, change, text):  # noqa: F811
    ctx, desc, lim, keep = _context()
    cache, seq, step = _state()
    args = dict(p=A, q=A, p_stride=4096, q_stride=4096, type=hs.HS_F32, u_accept=A, u_sample=A)
    _refused(lambda: hs.hs_accept_probs(ctx, hs.hs_accept_probs_args(**args), seq, step), hs.HS_ERR_CAPACITY, "workspace")
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    _refused(lambda: hs.hs_accept_probs(ctx, hs.hs_accept_probs_args(**args), hs.hs_seq_state(), step), hs.HS_ERR_INVALID_ARG, "sequence")
    _refused(lambda: hs.hs_accept_probs(ctx, hs.hs_accept_probs_args(**args), seq, hs.hs_step()), hs.HS_ERR_INVALID_ARG, "step")
    args.update(change)
    _refused(lambda: hs.hs_accept_probs(ctx, hs.hs_accept_probs_args(**args), seq, step), hs.HS_ERR_INVALID_ARG, text)
    hs.hs_destroy(ctx)
