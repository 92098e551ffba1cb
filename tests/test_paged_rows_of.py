"""What out-of-range numbers of a request mean, from the header that both paged attentions use, on the host (no GPU needed)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_numbers_out_of_range_are_clamped(tmp_path):
    exe = str(tmp_path / "rows")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2604_17397_amd", "csrc"), os.path.join(ROOT, "tests", "host", "paged_rows_of.cpp"),
                    "-o", exe], check=True)
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=100)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout
