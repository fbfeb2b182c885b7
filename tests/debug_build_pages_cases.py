"""Small cases of every call of the paged cache, run against the CHECKED build of the library (lib/libfaedkv_debug.so, selected
through FAEDKV_LIBRARY before this process starts).  Not collected by pytest: tests/test_gpu_pages_checked.py runs it in a
process of its own.  After every case the bounds-check word must be 0; the cases bring their canaries and references."""
import os
import sys

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
sys.path.insert(0, os.path.dirname(HERE))

import test_gpu_pages as cases                                       # noqa: E402
from paper_2507_20030_b200 import binding as fk                      # noqa: E402


def main():
    assert torch.cuda.is_available()
    assert fk.load().faedkv_debug_build() == 1, "this script must run against the checked build (FAEDKV_LIBRARY)"
    word = cases.make(fk).debug_word
    f32, bf16 = torch.float32, torch.bfloat16
    run = [(cases.test_tables, a) for a in [(1, 16, 4, 6, 2, 0), (7, 16, 20, 60, 50, 3), (7, 32, 3, 60, 200, 0), (300, 16, 9, 2000, 60, 5),
                                            (40, 128, 70, 2000, 3000, -100)]]
    run += [(cases.test_tables_flags_bad_lengths_and_stack, ()), (cases.test_store_of_values_at_the_edges, ()),
            (cases.test_store_skips_slots_outside_the_pool, ()), (cases.test_lengths_beyond_the_table_are_cut_and_reported, ())]
    for dtype in (bf16, f32):
        run += [(cases.test_store, (dtype, *a)) for a in [(16, 2, [16, 17, 40, 5], [16, 1, 23, 2]), (128, 2, [1000, 127, 129], [1000, 5, 2]),
                                                         (64, 8, [5000, 77], [4000, 77])]]
        run += [(cases.test_load, (dtype, *a)) for a in [(32, 3, [0, 100, 33], 101), (128, 4, [129, 500, 128], 700)]]
        run += [(cases.test_decode_attention, (dtype, *a)) for a in [(16, 2, 4, [127, 128, 129, 0, 1]), (64, 1, 5, [2500, 3])]]
        run += [(cases.test_ragged_causal_attention, (dtype, *a)) for a in [(16, 2, 4, [40, 9, 0, 3], [7, 9, 0, 1], 3), (16, 1, 2, [5], [9], 0),
                                                                           (64, 2, 4, [300, 128, 129], [130, 1, 129], 0)]]
        run += [(cases.test_attention_of_many_sequences, (dtype,)), (cases.test_a_served_run_against_the_reference, (dtype,))]
    run += [(cases.test_ragged_attention_over_split_caches, a) for a in [(64, 1, 4, [5000], [40]), (128, 8, 8, [900, 260], [100, 250])]]
    run += [(cases.test_attention_skips_pages_outside_the_pool, (new,)) for new in (None, [5], [90])]
    for case, args in run:
        case(fk, *args)
        torch.cuda.synchronize()
        w = word()
        assert w == 0, f"{case.__name__}{args}: bounds check failed, file tag {w >> 16} line {w & 0xffff}"
    print(f"checked build: {len(run)} paged cases ok")


if __name__ == "__main__":
    main()
