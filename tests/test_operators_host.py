"""What the operators in the 8-bit container compute on the way to their kernels, without a GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_34185_b200", "csrc")


def _program(tmp_path, source, *others):
    exe, nvcc = str(tmp_path / "program"), os.environ.get("NVCC") or "/usr/local/cuda/bin/nvcc"
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    "-o", exe, os.path.join(ROOT, "tests", source)] + list(others), check=True)
    return exe


def test_the_list_of_requests_is_their_running_sum(tmp_path):
    # with more requests than a CTA has threads a thread lays out several, and its counts may stand where the sums go
    calls, wrong = subprocess.run([_program(tmp_path, "request_list.cu")], check=True, capture_output=True, text=True, timeout=300).stdout.split()
    assert int(calls) > 3000 and wrong == "0"


def test_shares_of_prompts_take_every_tile_once_and_end_with_the_requests(tmp_path):
    program = _program(tmp_path, "prompt_shares.cu", os.path.join(CSRC, "stream.cpp"))
    assert subprocess.run([program], check=True, capture_output=True, text=True, timeout=300).stdout.split() == ["96", "0", "0", "0"]
