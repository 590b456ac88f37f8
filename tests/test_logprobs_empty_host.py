"""hs_logprobs about nothing: arrays without elements need no addresses, and what is wrong all the same is refused (no GPU)."""
import pytest

import paper_2508_18588_amd as hs
from test_boundary_host import lib  # noqa: F401  (the library fixture)
from test_more_operators_host import INVALID, _ask
from test_operators_host import _context, _refused, _state


@pytest.mark.parametrize("gone", [("logprob",), ("logits",), ("token", "row", "live"), ("entropy", "top_token", "top_logprob"),
                                  ("logits", "row", "token", "live", "logprob", "entropy", "top_token", "top_logprob")])
def test_arrays_of_no_elements(lib, gone):  # noqa: F811
    ctx, desc, lim, keep = _context()
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    hs.hs_logprobs(ctx, _ask(n=0, **{name: None for name in gone}))
    hs.hs_logprobs(ctx, _ask(n=0, rows=0, **{name: None for name in gone}))
    hs.hs_destroy(ctx)


@pytest.mark.parametrize("change,text", [(dict(temperature=0.0), "temperature"), (dict(top=-1), "top"), (dict(top=hs.HS_LOGPROBS_TOP + 1), "top"),
                                         (dict(logits_type=2), "type"), (dict(rows=-1), "rows"), (dict(logits_stride=4095), "stride")])
def test_what_is_wrong_is_refused(lib, change, text):  # noqa: F811
    ctx, desc, lim, keep = _context()
    _refused(lambda: hs.hs_logprobs(ctx, _ask(n=0, logprob=None)), hs.HS_ERR_CAPACITY, "workspace")
    hs.hs_bind_workspace(ctx, 0x100000, 1 << 40)
    _refused(lambda: hs.hs_logprobs(ctx, _ask(n=0, logprob=None, **change)), INVALID, text)
    # (emitted tokens: there is no n, and outputs are there)
    _refused(lambda: hs.hs_logprobs(ctx, _ask(n=0, emitted=1, logprob=None), *_state()[1:]), INVALID, "null output")
    hs.hs_destroy(ctx)
