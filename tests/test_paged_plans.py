"""The rule that picks the paged attention's kernel, on a machine without a GPU: the library's own C++ function, called through its
exported name.  0: the kernel of few rows, 1 or 2 Q tiles of the tensor cores', -1: refused."""
import ctypes

import pytest


def kernel(n_seqs, max_rows, max_new, group, kv_heads, longest, out_stride=4096):
    from paper_2511_21759_b200 import binding as B
    f = B.lib()._ZN3odb25paged_attention_kernel_ofEiiiiixx
    f.argtypes, f.restype = [ctypes.c_int] * 5 + [ctypes.c_longlong] * 2, ctypes.c_int
    return f(n_seqs, max_rows, max_new, group, kv_heads, longest, out_stride)


@pytest.mark.parametrize("n_seqs,max_rows,max_new,group,kv_heads,longest,want", [
    (1, 1, 1, 4, 8, 640, 0), (48, 48, 1, 4, 8, 8192, 0), (2, 2, 1, 4, 8, 131072, 0),          # single tokens
    (16, 512, 32, 4, 8, 4096, 1), (16, 512, 32, 4, 8, 64, 1), (2, 64, 32, 4, 8, 64, 0),       # blocks; little work
    (1, 4096, 4096, 4, 8, 4096, 2), (4, 4900, 1536, 1, 32, 1536, 2),                          # prompts that are alike
    (48, 2095, 2048, 4, 8, 8192, 1), (9, 4104, 4096, 4, 8, 8192, 1),                          # one among single tokens
    (1, 4096, 4096, 130, 1, 4096, 0), (1, 4096, 4096, 128, 1, 4096, 2),                       # a group that no Q tile holds
])
def test_kernel_of_requests(n_seqs, max_rows, max_new, group, kv_heads, longest, want):
    assert kernel(n_seqs, max_rows, max_new, group, kv_heads, longest) == want


@pytest.mark.parametrize("n_seqs,max_rows,max_new,group,kv_heads,longest,want", [
    (1, 131072, 131072, 4, 8, 131072, 2), (1, 262144, 262144, 4, 8, 262144, 2), (1, 1000000, 1000000, 4, 8, 1000000, 2),
    (1, 262144, 1, 4, 8, 262144, 1),                                  # the hint says few rows, whose kernel has no 32-bit numbers for them
    (1, 700000, 1, 4, 8, 1000000, 2),                                 # nor has one Q tile
    (1, 1 << 20, 1 << 20, 4, 8, 1 << 20, -1), (1, 1 << 20, 1, 4, 8, 1 << 20, -1),
    (1, 1 << 14, 1 << 14, 130, 1, 1 << 14, 0),
    (1, 1 << 18, 1 << 18, 130, 1, 1 << 18, -1),
    (1024, 1024, 1, 1, 1, 1 << 20, 0),
])
def test_every_prompt_is_taken_that_some_kernel_can_count(n_seqs, max_rows, max_new, group, kv_heads, longest, want):
    """Sums of key tiles over a launch's items are 32-bit numbers; the larger a kernel's items the fewer of them."""
    assert kernel(n_seqs, max_rows, max_new, group, kv_heads, longest) == want


def test_rows_far_apart_take_the_kernel_of_few_rows():
    at = lambda stride: kernel(1, 4096, 4096, 4, 8, 4096, stride)
    assert at(1 << 27) == 2 and at((1 << 27) + 8) == 0 and at(1 << 40) == 0


@pytest.mark.parametrize("n_seqs,max_rows,group,want", [
    (48, 48, 4, 0), (16, 64, 4, 0), (16, 65, 4, 1),                   # the mean stands for the longest: few rows or many
    (1, 4096, 4, 2), (1, 4096, 1, 2), (1, 33, 4, 2), (1, 20, 4, 1),   # one request: the mean is the longest
    (48, 2048 + 47, 4, 1), (16, 512 + 15, 4, 1), (16, 2048, 4, 1),    # fewer than 1024 packed rows on average: one Q tile
    (16, 4096 + 15, 4, 2), (4, 4096, 4, 2), (8, 8 * 256, 4, 2), (4, 4096, 1, 2), (5, 4096, 1, 1),
])
def test_kernel_of_requests_whose_longest_is_not_known(n_seqs, max_rows, group, want):
    assert kernel(n_seqs, max_rows, 0, group, 8, 8192) == want
