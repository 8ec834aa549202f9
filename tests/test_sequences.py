"""The ragged sequences of a call on the cache, on the host: tests/sequences.cpp, built with the library's header."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_tiles_rows_and_pages(tmp_path):
    made = str(tmp_path / "sequences")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2410_20650_amd", "csrc"), os.path.join(ROOT, "tests", "sequences.cpp"), "-o", made], check=True)
    done = subprocess.run([made], capture_output=True, text=True)
    assert done.returncode == 0 and done.stdout == "ok\n", done.stdout + done.stderr
