"""CPU-only: the smoke run's cases take no launch that a profiler cannot replay."""
import __graft_entry__ as entry


def test_no_fp32_case_takes_the_cooperative_launch():
    """64 keys are a tile of the fp32 kernels; windows that straddle tiles take two ordinary launches (test_launch_rules.py), whole ones a cooperative launch."""
    cases = entry.smoke_workloads()
    assert sorted(w.dtype for w in cases) == ["bf16", "f32"]
    for w in cases:
        assert w.dtype == "bf16" and w.head_dim in (64, 128) or 64 % w.window != 0
