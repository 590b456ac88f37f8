"""hs_set_window and hs_attention_window from Python: numbers that do not fit their 32 bits are refused and not cut (no GPU)."""
import pytest

import paper_2508_18588_amd as hs
from test_boundary_host import lib  # noqa: F401  (the library fixture)
from test_operators_host import A, _context


@pytest.mark.parametrize("big", [2 ** 32 + 16, 2 ** 31 + 5, -2 ** 32 + 7, 2 ** 64 + 1])
def test_windows_and_sinks_beyond_32_bits(lib, big):  # noqa: F811
    ctx, desc, lim, keep = _context()
    with pytest.raises(ValueError, match="window"):
        hs.hs_set_window(ctx, [16, big], 4)
    with pytest.raises(ValueError, match="sinks"):
        hs.hs_set_window(ctx, [16, 0], big)
    hs.hs_destroy(ctx)


@pytest.mark.parametrize("name", ["layer", "window", "sinks", "chunk"])
@pytest.mark.parametrize("big", [2 ** 32 + 1, -2 ** 32 + 1])
def test_attention_window_beyond_32_bits(lib, name, big):  # noqa: F811
    args = dict(layer=0, window=8, sinks=4, chunk=1, q=A, out=A)
    hs.hs_window_args(**args)
    with pytest.raises(ValueError, match=name):
        hs.hs_window_args(**dict(args, **{name: big}))
