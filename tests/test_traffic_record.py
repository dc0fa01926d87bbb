"""The benchmark's record of DRAM traffic: a figure counts while the files that its kernel is compiled from are those of its
capture, and files that the kernel does not include have no say."""
import os
import shutil

import bench


def record(tmp_path, line):
    path = tmp_path / "record.txt"
    path.write_text("# figures\n" + line + "\n")
    return str(path)


def test_hash_covers_what_a_kernel_includes(tmp_path):
    csrc = str(tmp_path / "csrc")
    shutil.copytree(bench.CSRC, csrc)
    h = bench.kernel_source_hash("roi_fwd.cu", csrc)
    assert h == bench.kernel_source_hash("roi_fwd.cu") and h != bench.kernel_source_hash("roi_bwd.cu")
    line = f"kernel=roi_fwd_kernel<2,4,tau1> file=roi_fwd.cu sources={h} dram_bytes_per_element=7.5 capture=1x4"
    traffic = lambda tag="roi_fwd_kernel<2,4,tau1>": bench.recorded_traffic(tag, record(tmp_path, line), csrc)  # noqa: E731
    assert traffic() == 7.5 and traffic("roi_bwd_kernel<2,4,tau1>") is None
    # another kernel's file, and a new one
    for name in ("roi_optim.cu", "roi_fp8.cuh", "roi_new.cu"):
        with open(os.path.join(csrc, name), "a") as f:
            f.write("// more\n")
        assert traffic() == 7.5, name
    # a header of a header that it includes
    with open(os.path.join(csrc, "roi_vec.cuh"), "a") as f:
        f.write("// more\n")
    assert traffic() is None


def test_records_without_their_file_do_not_count(tmp_path):
    line = "kernel=k sources=0123456789abcdef dram_bytes_per_element=7.5"
    assert bench.recorded_traffic("k", record(tmp_path, line)) is None
    assert bench.recorded_traffic("k", record(tmp_path, line + " file=none.cu")) is None


def test_every_record_names_its_file():
    with open(os.path.join(bench.ROOT, "profiles", "dram_traffic.txt")) as f:
        lines = [ln for ln in f if ln.strip() and not ln.startswith("#")]
    assert len(lines) == 9
    for ln in lines:
        kv = dict(x.split("=", 1) for x in ln.split() if "=" in x)
        with open(os.path.join(bench.CSRC, kv["file"])) as f:
            text = f.read()
        name = kv["kernel"].split("<")[0]
        assert name in text or name.replace("roi_", "roi_slice_") in text
