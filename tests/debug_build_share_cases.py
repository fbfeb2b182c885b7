"""Small cases of shared pages and differential attention, run against the CHECKED build of the library (lib/libfaedkv_debug.so, selected
through FAEDKV_LIBRARY before this process starts).  Not collected by pytest: tests/test_gpu_pages_share_checked.py runs it in a process of its
own.  After every case the bounds-check word must be 0."""
import os
import sys

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
sys.path.insert(0, os.path.dirname(HERE))

import test_gpu_pages_diff as diff                                   # noqa: E402
import test_gpu_pages_share as share                                 # noqa: E402
import test_gpu_pages_shared as shared                               # noqa: E402
from paper_2507_20030_b200 import binding as fk                      # noqa: E402


def main():
    assert torch.cuda.is_available()
    assert fk.load().faedkv_debug_build() == 1, "this script must run against the checked build (FAEDKV_LIBRARY)"
    word = share.make(fk).debug_word
    f32, bf16 = torch.float32, torch.bfloat16
    run = [(share.test_fork, (*a, cut)) for cut in (False, True) for a in [(1, 16, 1, 2, 1, False), (5, 32, 40, 30, 20, True), (1, 16, 2, 2600, 2400, True)]]
    run += [(share.test_fork_refuses_rows_that_cannot_be_written, ()), (share.test_fork_flags_bad_pages_lengths_and_stack, ()),
            (share.test_release_flags_what_is_out_of_range, ()), (share.test_compact_flags_pages_outside_the_pool, ()),
            (share.test_requests_that_share_pages_live_and_end, ())]
    run += [(share.test_release, a) for a in [(16, 30, 7, 200), (32, 3, 3000, 6000), (16, 9, 30, 65537)]]
    run += [(share.test_compact, a) for a in [(2, 16, 9, 6, 100), (8, 64, 12, 30, 700), (1, 16, 50, 1500, 66000)]]
    for dtype in (bf16, f32):
        run += [(shared.test_groups, (dtype, *a)) for a in [(16, 2, 4, [(128, [128, 129, 128, 200, 131])]), (32, 1, 7, [(960, [1000] * 11), (0, [77]), (32, [33, 64])]),
                                                            (128, 2, 8, [(256, [300, 256]), (128, [1000, 129, 128, 500])])]]
        run += [(shared.test_rows_shorter_than_their_group, (dtype,)), (shared.test_empty_groups_and_rows_of_no_group, (dtype,)),
                (shared.test_nan_and_missing_pages, (dtype,)), (shared.test_more_blocks_than_are_shared_out, (dtype,))]
        run += [(diff.test_decode, (dtype, *a, gain)) for gain in (True, False) for a in [(32, 2, 4, [127, 128, 129, 0, 1]), (16, 1, 2, [2500, 3])]]
        run += [(diff.test_new_tokens, (dtype, *a)) for a in [(16, 2, 4, [40, 9, 0, 3], [7, 9, 0, 1], 3), (64, 2, 2, [300, 128, 129], [130, 1, 129], 0),
                                                             (16, 1, 2, [5], [9], 0)]]
    run += [(shared.test_groups_of_many_columns, a) for a in [(16, 1, 8, [(2048, [2050] * 33)]), (32, 5, 2, [(1600, [1601 + i for i in range(64)])])]]
    run += [(diff.test_new_tokens_over_split_caches, a) for a in [(64, 1, 4, [5000], [40]), (16, 2, 2, [3000, 700], [20, 3])]]
    run += [(diff.test_nan_reaches_the_rows_that_see_it, (k,)) for k in (0, 1)]
    for case, args in run:
        case(fk, *args)
        torch.cuda.synchronize()
        w = word()
        assert w == 0, f"{case.__name__}{args}: bounds check failed, file tag {w >> 16} line {w & 0xffff}"
    print(f"checked build: {len(run)} cases of shared pages ok")


if __name__ == "__main__":
    main()
