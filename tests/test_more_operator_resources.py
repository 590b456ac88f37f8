"""Register and LDS budgets of the shared attention's, the log probabilities' and the pages' kernels, from the compiler's resource report (no GPU)."""
from test_kernel_resources import resource_report


def test_shared_attention_keeps_two_workgroups_per_compute_unit():
    rep = resource_report("hs_shared.hip")
    assert len(rep) == 6, sorted(rep)                          # walks per head size; joins per head size, with few rows and many
    for name, r in rep.items():
        if "shared_rows" in name:
            assert r["Occupancy [waves/SIMD]"] >= 2 and r["LDS Size [bytes/block]"] <= 80 * 1024, (name, r)
            assert r["VGPRs Spill"] <= 8, (name, r)            # (a few words, in front of the loops over keys)
        else:
            assert r["ScratchSize [bytes/lane]"] == 0 and r["VGPRs Spill"] == 0, (name, r)


def test_log_probabilities_and_pages_use_no_scratch():
    rep = {**resource_report("hs_logprobs.hip"), **resource_report("hs_pages.hip")}
    assert len(rep) == 4 + 10, sorted(rep)
    for name, r in rep.items():
        assert r["ScratchSize [bytes/lane]"] == 0 and r["VGPRs Spill"] == 0, (name, r)
        assert r["Occupancy [waves/SIMD]"] >= 4, (name, r)
