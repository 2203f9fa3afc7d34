"""What the entry points for a vocabulary's logits launch at their largest sizes, on the host (tests/_launched.py)."""
from tests._launched import launched


def _distill(B, V, dtype):
    p = "@256"
    return "distill_xent", [dtype, B, V, 4, p, V, p, p, None, None, 1.0, 1.0 / B, p, p, None, 0, dtype, p, 1 << 40, None]


def test_rows_of_large_workgroups_stay_within_a_launch():
    """A launch holds fewer than 2^32 work-items: rows that take 512 or 1024 threads each go in parts, of 256, from 2^23 or
    2^22 rows on."""
    rows, parts = "distill_xent", "distill_xent (sums)"
    cases = [(2 ** 24 - 1, 16391, 1, rows), (2 ** 24 - 1, 8195, 0, rows), (2 ** 23 - 1, 16392, 1, rows), (2 ** 23, 16392, 1, parts),
             (2 ** 23 - 1, 16384, 0, rows), (2 ** 23, 16384, 0, parts), (2 ** 24 - 1, 32768, 1, parts), (2 ** 22 - 1, 32776, 1, rows),
             (2 ** 22, 32776, 1, parts), (2 ** 22 - 1, 131072, 1, rows), (2 ** 22, 131072, 1, parts), (2 ** 22, 16388, 0, parts),
             (4096, 131072, 1, rows), (4096, 50021, 0, rows)]
    assert launched([_distill(*c[:3]) for c in cases]) == [c[3] for c in cases]
