"""Which sources a counter summary of the benchmark's kernel belongs to (no GPU)."""

import bench


def test_the_kernel_s_own_sources():
    """Its unit and that unit's headers; a change to the calls around a verification does not make its counters stale."""
    assert sorted(bench.kernel_sources()) == ["mpv.hip", "mpv_device.h", "mpv_exchange.h", "mpv_nucleus.h"]
    assert len(bench.kernel_source_digest()) == 16


def test_counters_of_other_sources_are_not_reported(tmp_path):
    for sources, want in ((bench.kernel_source_digest(), 5.0), ("0" * 16, None)):
        path = tmp_path / "counters.txt"
        path.write_text(f"# read\nhbm_bytes_per_launch = 5.0\nkernel_sources_sha256_16 = {sources}\n")
        traffic, provenance = bench.parse_profile_traffic(str(path))
        assert traffic == want and provenance["status"].startswith("current" if want else "stale")
