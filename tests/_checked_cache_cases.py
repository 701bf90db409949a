"""The cache's tests run against the bounds-checked build (liboccam_checked.so): each ends with
device status 0 (no index outside its buffer), or with the error that it expects. Run as a script in
its own process (the binding loads one library per process); exits non-zero on any failure."""

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
    import test_gpu_cache as T

    assert "liboccam_checked.so" in occ.library()._name
    cases = [
        (T.test_append, ("bf16", 16, 64, 2)), (T.test_append, ("f16", 128, 128, 1)), (T.test_append_many_sequences_and_rows_outside, ()),
        (T.test_pages, (16, 64, 2, 3)), (T.test_pages, (64, 128, 5, 2)), (T.test_pages_many_sequences, ()),
        (T.test_offsets_past_32_bits, ()), (T.test_device_errors_change_nothing, ()),
        (T.test_append_behind_a_refused_extend_changes_nothing, ()), (T.test_append_writes_no_shared_page, ()),
        (T.test_attend_many_sequences, ()), (T.test_attend_long_caches_mostly_hidden, (16, 128, 7)),
        (T.test_attend_long_caches_mostly_hidden, (128, 64, 70)), (T.test_streams_and_graph, ()),
    ]
    cases += [(T.test_attend, (n, "bf16")) for n in range(len(T.ATTEND))]
    cases += [(T.test_attend_hidden_tokens, (n, n % 2 == 0)) for n in range(len(T.ATTEND))]
    cases += [(T.test_attend_long_splits_many_ways, (rows,)) for rows in ([1, 1, 1], [20, 1, 300])]
    for f, args in cases:
        f(*args)
        print("ok", f.__name__, args, flush=True)
    print("done", len(cases), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
