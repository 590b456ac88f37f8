"""Register and LDS budgets of the window attention's and the probabilities' kernels, from the compiler's resource report (no GPU)."""
import pytest

from test_kernel_resources import resource_report


@pytest.fixture(scope="module")
def window():
    return resource_report("hs_window.hip")


def test_window_attention_keeps_two_workgroups_per_compute_unit(window):
    """Registers for two wavefronts per SIMD, LDS for two rings; what is spilled is a few words, in front of the loops over keys."""
    hot = {k: v for k, v in window.items() if "window_rows" in k or "window_chunk" in k}
    assert len(hot) == 8, sorted(window)                       # few rows, ring (whole and in parts), chunks; head sizes 64 and 128
    for name, r in hot.items():
        assert r["Occupancy [waves/SIMD]"] >= 2 and r["LDS Size [bytes/block]"] <= 80 * 1024, (name, r)
        assert r["VGPRs Spill"] <= 8, (name, r)


def test_few_rows_and_merge_use_no_scratch(window):
    cold = {k: v for k, v in window.items() if "window_merge" in k or "window_rowsI" in k}
    assert len(cold) == 6, sorted(window)
    for name, r in cold.items():
        assert r["ScratchSize [bytes/lane]"] == 0 and r["VGPRs Spill"] == 0, (name, r)


def test_probabilities_and_verification_use_no_scratch():
    rep = resource_report("hs_probs.hip")
    assert len(rep) == 14, sorted(rep)                         # rows and writes per pair of types, statistics, sums and picks per type
    for name, r in rep.items():
        assert r["ScratchSize [bytes/lane]"] == 0 and r["VGPRs Spill"] == 0, (name, r)
        if "verify" not in name:
            assert r["Occupancy [waves/SIMD]"] >= 4, (name, r)      # a workgroup of 1024 threads, or eight of 256
