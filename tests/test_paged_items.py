"""The numbering of paged attention's workgroups on the host (no GPU needed)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_pair_of_tiles_is_one_items_and_every_piece_has_its_slot(tmp_path):
    exe = str(tmp_path / "items")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2604_17397_amd", "csrc"), os.path.join(ROOT, "tests", "host", "paged_attn_items.cpp"),
                    "-o", exe], check=True)
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout
