"""What a context's workspace takes: shared prefixes borrow arrays that are idle while attention runs (no GPU)."""
import ctypes as C

import pytest

import paper_2508_18588_amd as hs
from test_boundary_host import lib  # noqa: F401  (the library fixture)

SHAPES = {"toy": (2, 256, 4, 4, 64, 1024, 4096), "1.5b": (28, 1536, 12, 2, 128, 8960, 151936), "7b": (28, 3584, 28, 4, 128, 18944, 152064),
          "14b": (48, 5120, 40, 8, 128, 13824, 152064)}


def workspace(shape, batch, k_max, c_max, rows, blocks):
    d = SHAPES[shape]
    arr = (C.c_void_p * d[0])(*[0x1000] * d[0])
    p = C.cast(arr, C.POINTER(C.c_void_p))
    w = hs.hs_weights(0x1000, 0x1000, 0x1000, p, p, p, p, p, p, p, 0x1000)
    ctx = hs.hs_create(hs.hs_model_desc(*d, 16, 1e-6), w, hs.hs_limits(batch, k_max, c_max, rows, blocks, 16 * blocks, 8))
    n = hs.hs_workspace_bytes(ctx)
    hs.hs_destroy(ctx)
    return n


@pytest.mark.parametrize("shape,limits,without", [
    # limits: sequences, k_max, c_max, rows, pages per sequence; bytes that the same context needs for all other calls
    ("1.5b", (64, 8, 2, 16384, 560), 4747430656), ("1.5b", (16, 4, 1, 16384, 256), 3760810752),
    ("7b", (128, 16, 1, 2304, 256), 667659264), ("7b", (64, 8, 2, 16384, 560), 5941373696), ("7b", (256, 8, 1, 16384, 2048), 7639449088),
    ("14b", (128, 16, 1, 2176, 256), 614012928), ("14b", (64, 8, 2, 16384, 560), 5469514496), ("14b", (16, 4, 1, 16384, 256), 6680275712),
    ("toy", (64, 8, 2, 16384, 560), 360683264),
])
def test_large_contexts_hold_no_memory_for_prefixes_that_they_do_not_share(lib, shape, limits, without):  # noqa: F811
    """But for the log probabilities' 16 MB, a number per sequence and what a few arrays more are rounded up by."""
    assert workspace(shape, *limits) <= without + (16 << 20) + 4096


@pytest.mark.parametrize("shape", list(SHAPES))
def test_small_contexts_hold_room_for_a_useful_call(lib, shape):  # noqa: F811
    """With few rows there is little to borrow: room for many runs of a prefix, 64 MB and their sums at most, and for 16 MB of log probabilities."""
    for batch in (1, 4, 128):
        assert 16 << 20 <= workspace(shape, batch, 0, 1, batch, 512) < 128 << 20
