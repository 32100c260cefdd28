"""The summary of a kernel trace by launch shape (no GPU)."""
import sys

import bench
from paper_2608_14376_amd import prof_summary

HEAD = ("Kernel_Name,Start_Timestamp,End_Timestamp,Grid_Size_X,Grid_Size_Y,Grid_Size_Z,"
        "Workgroup_Size_X,Workgroup_Size_Y,Workgroup_Size_Z\n")


def test_launches_are_grouped_by_kernel_and_shape(tmp_path, monkeypatch):
    row = '"void ns::(anonymous namespace)::%s(float*, int)",%d,%d,%d,%d,1,256,1,1\n'
    trace, out = tmp_path / "t.csv", tmp_path / "s.txt"
    trace.write_text(HEAD + row % ("k_two<64>", 9000, 12000, 512, 1) + row % ("k_one<128, true>", 1000, 2000, 2048, 5) +
                     row % ("k_one<128, true>", 3000, 7000, 2048, 5) + row % ("other", 100, 200, 256, 1) +
                     row % ("k_one<128, true>", 8000, 8500, 256, 1))
    monkeypatch.setattr(sys, "argv", ["prof_summary", "launches", "--trace", str(trace), "--out", str(out), "--title", "a title",
                                      "--command", "a command", "--source", "cache.hip", "--source", "cache.h"])
    prof_summary.main()
    lines = out.read_text().splitlines()
    assert lines[0] == "# a title" and lines[1] == "# command: a command"
    assert bench.read_summary(str(out))["kernel_source_sha256_16"] == prof_summary.source_sha(("cache.hip", "cache.h"))
    table = [ln.split() for ln in lines if ln.startswith("k_")]
    assert table == [["k_one<128,", "true>", "8", "x", "5", "x", "1", "256", "2", "1.00", "4.00", "4.00"],
                     ["k_one<128,", "true>", "1", "x", "1", "x", "1", "256", "1", "0.50", "0.50", "0.50"],
                     ["k_two<64>", "2", "x", "1", "x", "1", "256", "1", "3.00", "3.00", "3.00"]]
