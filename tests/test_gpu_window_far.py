"""Window attention of sequences that have grown far beyond their block table: the table's positions are seen as far as the rows' windows
reach back into them, and the sinks; whole walks, wavefronts' and workgroups' partitions, chunks and the plain kernel."""
import numpy as np
import pytest
import torch

from window_common import chain, check, engine, lay_out, lay_out_chunk, queries, reference

pytestmark = pytest.mark.gpu

# heads, sequences, positions of the longest text, nodes: how a draft's keys are taken follows from these and the window
SIZES = [((8, 1, 64), 3, 80, 5), ((8, 1, 128), 3, 470, 4), ((8, 1, 128), 3, 470, 9), ((14, 2, 64), 2, 470, 9), ((8, 1, 64), 256, 470, 9)]


def run(eng, m, q, window, sinks, chunk=0):
    out = torch.full((eng.max_rows, q.shape[1]), 7.0, device="cuda:0", dtype=q.dtype)
    full = torch.zeros(eng.max_rows, q.shape[1], device="cuda:0", dtype=q.dtype)
    full[:m] = q
    if eng.workspace is not None:
        eng.workspace.fill_(0xFF)                            # (partial results of nobody: NaNs)
    eng.attention_window(0, full, out, window, sinks, chunk)
    torch.cuda.synchronize()
    assert (out[m:] == 7.0).all()
    return out


class grown:
    """The engine with a table that goes on (of whose further pages the reference is to see nothing)."""

    def __init__(self, eng, most):
        self.eng, self.table = eng, eng.block_table
        self.wide = torch.cat([eng.block_table, eng.block_table[:, :1].expand(-1, most // 16 + 2)], 1)

    def __enter__(self):
        self.eng.block_table = self.wide

    def __exit__(self, *a):
        self.eng.block_table = self.table


@pytest.mark.parametrize("heads,batch,longest,nodes", SIZES)
@pytest.mark.parametrize("window,sinks", [(1, 4), (50, 0), (50, 4), (200, 0), (300, 70), (4096, 0)])
def test_far_beyond_the_table(heads, batch, longest, nodes, window, sinks):
    eng = engine(*heads, [longest] + [33] * (batch - 1), nodes)
    cap = eng.block_table.shape[1] * 16
    for chunk in (0, nodes):
        for beyond in (1, 11, 41, 201, 333, 5000) if batch < 9 else (41, 333):
            lens = [cap + beyond] + [33] * (batch - 1)
            eng.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
            pars = [chain(nodes - 1)] * 2 + [chain(0)] * (batch - 2)
            m = lay_out_chunk(eng, [len(p) for p in pars]) if chunk else lay_out(eng, lens, pars)
            q = queries(m, eng)
            out = run(eng, m, q, window, sinks, chunk)
            with grown(eng, max(lens) + nodes):
                check(out, eng, lens, pars, q, window, sinks, chunk=bool(chunk), blocked=lambda b: np.arange(max(lens) + nodes) >= cap)
            if sinks == 0 and beyond > window:               # nothing is left of the windows
                assert (out[:nodes] == 0).all()
    eng.close()


@pytest.mark.parametrize("heads,batch,longest,nodes", SIZES)
def test_the_longest_sequence_there_can_be(heads, batch, longest, nodes):
    """Positions just below 2^31: what is left is the sinks, with the bits of any other sequence that has left its table behind."""
    eng = engine(*heads, [longest] + [33] * (batch - 1), nodes)
    cap = eng.block_table.shape[1] * 16
    for window, sinks, chunk in ((100, 70, 0), (1 << 30, 5, 0), (100, 0, 0), (100, 70, nodes), (1 << 30, 5, nodes)):
        outs = []
        for first in (cap + window + 1, 2 ** 31 - 1 - nodes):
            lens = [first] + [33] * (batch - 1)
            eng.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
            pars = [chain(nodes - 1)] * batch
            m = lay_out_chunk(eng, [nodes] * batch) if chunk else lay_out(eng, lens, pars)
            outs.append(run(eng, m, queries(m, eng), window, sinks, chunk))
        assert torch.isfinite(outs[0].float()).all() and torch.equal(outs[0], outs[1])
        assert (outs[0][:nodes] == 0).all() == (sinks == 0)
    eng.close()


def test_the_plain_kernel_far_beyond_the_table():
    eng = engine(8, 2, 64, [80, 33], 5, precise=True)
    cap = eng.block_table.shape[1] * 16
    for beyond in (1, 11, 41, 201):
        lens, pars = [cap + beyond, 33], [chain(4), chain(0)]
        eng.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        m = lay_out(eng, lens, pars)
        q = queries(m, eng)
        for window, sinks in ((1, 4), (50, 0), (50, 4), (4096, 0)):
            got = run(eng, m, q, window, sinks)[:m].double()
            with grown(eng, max(lens) + 5):
                want, mag = reference(eng, lens, pars, q, window, sinks, blocked=lambda b: np.arange(max(lens) + 5) >= cap)
            # (products, exponentials and sums in 64 bits, the scale in 32: as without a table that ends)
            assert ((got - want).abs() <= 2.0 ** -24 * want.abs() + 2e-6 * mag + 1e-12).all(), (beyond, window, sinks)
    eng.close()
