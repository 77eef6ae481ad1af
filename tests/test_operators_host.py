"""What the operators in the 8-bit container compute on the way to their kernels, without a GPU."""
import os
import subprocess

import torch

import paper_2609_34185_b200 as ep

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


def test_strides_of_a_single_row_or_head_mean_nothing():
    # a step of one token comes out of products and slices with whatever stride: only what lies between rows that exist counts
    heads, matrix, bf = ep.binding._heads, ep.binding._matrix, torch.bfloat16
    one = torch.zeros(128, dtype=bf).as_strided((1, 2, 64), (1, 64, 1))
    assert one.stride() == (1, 64, 1) and heads(one, bf, one.shape, -1, "k") == (0, 64)
    single = torch.zeros(9, 67, dtype=bf)[:, None, :64]
    assert single.stride() == (67, 67, 1) and heads(single, bf, single.shape, -1, "k") == (67, 0)
    assert heads(torch.zeros(3, 2, 72, dtype=bf)[:, :, :64], bf, (3, 2, 64), -1, "k") == (144, 72)
    for t, ld in ((torch.zeros(5, 264)[:1, :256], 256), (torch.zeros(256, 1).t(), 256), (torch.zeros(1, 100), 112), (torch.zeros(0, 48), 48), (torch.zeros(5, 264)[:2, :256], 264)):
        assert matrix(t, torch.float32, t.shape, -1, "x") == ld


def test_the_status_of_bad_pages_names_both_its_causes():
    assert "page number outside the cache" in ep.strerror(-9) and "several requests" in ep.strerror(-9)


def test_work_beyond_64_bits_is_refused():
    # 2^22 units of tokens x 2^27 tiles of rows x 2^15 heads are 2^64 pieces of work, which 64 bits hold as none
    p = 1 << 20                                           # an address that is never read
    job = lambda N, heads, columns: ep.binding.ATTENTION_JOB.pack(p, p, p, p, 1, heads, 16, 64, p, p, p, columns, columns, 1, N, p, p, 0, p, 1 << 40, 64, 64, 64, 64, 1.0, heads, ep.BF16, 1)  # noqa: E731
    assert ep.load().ep_cache_attention(job(2 ** 31 - 16, 2 ** 15, 2 ** 26), None) == -3
    assert ep.load().ep_cache_attention(job(2 ** 31 - 1, 2 ** 15, 2 ** 26), None) == -3
    assert ep.load().ep_cache_attention(job(2 ** 31 - 1, 1, 2 ** 8), None) == -3
