"""The note beside bench.py's profiled figures names the library that was profiled, not the one that runs."""
import json

from test_bench_provenance import bench


def test_the_note_names_the_profiled_version(tmp_path):
    b = bench()
    path = str(tmp_path / "figures.txt")
    with open(path, "w") as f:
        json.dump({"sources": b.kernel_sources_hash(), "hbm_bytes_per_launch": 7.0, "valu_busy_frac": 0.5, "library_version": 17, "source": "x"}, f)
    note = b.profiled_traffic(path, 23)[2]
    assert "library version 17" in note and "library version 23" not in note
