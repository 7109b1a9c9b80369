"""The bench line's DRAM traffic: the committed capture belongs to the GEMM's present sources (no GPU)."""
import bench


def test_the_capture_is_of_the_present_sources():
    traffic, note = bench.traffic_record("k_tc_gemm_step", "falcon180b_down_14848x59392")
    assert traffic is not None, note
    assert 1e9 < traffic < 1e10                          # 2321 launches of one step


def test_other_workloads_have_none():
    assert bench.traffic_record("k_tc_gemm_step", "no such layer") == (None, "no committed capture for this workload")
