"""The tests of whole-prompt attention, its gradient, append with the rotation and attention over shared pages run against
the bounds-checked build (liboccam_checked.so): each ends with device status 0 (no index outside its
buffer), or with the error that it expects. Run as a script in its own process; exits non-zero on any failure."""

from __future__ import annotations

import os
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path[:0] = [os.path.dirname(HERE), HERE]


def main() -> int:
    from paper_2605_29657_gb300 import _lib as L
    from paper_2605_29657_gb300 import build as pb

    L.use_library(pb.LIB_CHECKED)
    import paper_2605_29657_gb300 as occ
    import test_gpu_append_rope as A
    import test_gpu_attend_shared as S
    import test_gpu_cache_short as C
    import test_gpu_prompt as P
    import test_gpu_prompt_grad as G
    import test_gpu_prompt_grad_parts as GP
    import test_gpu_prompt_serving as V

    assert "liboccam_checked.so" in occ.library()._name
    cases = [(P.test_prompt, (n, ("bf16", "f16")[n % 2])) for n in range(len(P.CASES))]
    cases += [(G.test_grad, (n, ("f16", "bf16")[n % 2])) for n in range(len(P.CASES))]
    cases += [(GP.test_grad_of_few_key_heads, (n, ("bf16", "f16")[n % 2])) for n in range(len(GP.PARTS))]
    cases += [(S.test_attend_shared, (n, "bf16")) for n in range(len(S.SHARED))]
    cases += [(S.test_attend_shared_where_it_pays, (n, "f16")) for n in range(len(S.PAYS))]
    cases += [
        (P.test_prompt_without_keys, ()), (P.test_prompt_many_sequences, ()), (P.test_prompt_offsets_that_do_not_fit_are_recorded, ()),
        (G.test_grad_without_keys, ()), (G.test_grad_many_sequences, ()), (G.test_grad_offsets_that_do_not_fit_are_recorded, ()),
        (A.test_append_rope, (16, 64, 2, 2, 64, "half", "bf16")), (A.test_append_rope, (64, 128, 3, 6, 64, "adjacent", "f16")),
        (A.test_append_rope, (128, 128, 1, 1, 128, "half", "bf16")), (A.test_append_rope_many_sequences_and_rows_outside, ()),
        (G.test_grad_of_many_items_of_one_step, (4, 2, 64, "bf16")), (G.test_grad_of_many_items_of_one_step, (3, 3, 128, "f16")),
        (G.test_grad_of_rows_that_see_one_key, (3, "bf16")), (GP.test_grad_parts_beside_a_sequence_that_does_not_fit, ([1000, 2000, 0, 1000], None, "f16")),
        (A.test_append_offsets_that_go_back_are_recorded, ([0, 640, 0, 640], 300)),
        (A.test_append_rope_of_many_conversations, (256,)), (A.test_append_rope_of_many_conversations, (700,)),
        (A.test_append_rope_many_heads_share_a_page, ()), (A.test_append_rope_errors_change_nothing, ()),
        (S.test_attend_shared_whatever_the_groups, ()), (S.test_attend_shared_device_errors, ()),
        (C.test_attend_many_short_items, (30, 150, 9, 32)), (V.test_prompts_enter_fork_and_answer, (64, 128, 2, 4, [150, 70, 301], 3, "bf16")),
        (V.test_rows_far_apart, ()),
    ]
    for f, args in cases:
        f(*args)
        print("ok", f.__name__, args, flush=True)
    print("done", len(cases), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
