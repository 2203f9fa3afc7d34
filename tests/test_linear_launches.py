"""Which kernel takes a layer's product, on the host (tests/_launched.py). The cases are those that tests/test_gpu_linear_exact.py
computes on the GPU, so that a kernel that it is meant to reach does not move away from it unseen."""
import pytest

from tests._launched import launched

ROWS, SKINNY, WIDE, TILE, PAIR = "linear_rows", "linear_skinny", "linear_wide", "linear_tile", "linear_pair"

# product(s), type, rows, d_out, d_in; the kernel, whether K is cut into ranges, copies padded to whole 16-byte chunks
CASES = [
    # large tiles, of 128 and of 256 rows; ranges of K; short of whole tiles on both sides
    ("fwd", "bf16", 2600, 2568, 2056, WIDE, False, 0), ("fwd", "bf16", 3001, 4104, 520, WIDE, False, 0),
    ("fwd", "bf16", 520, 4104, 4104, WIDE, True, 0), ("fwd", "bf16", 200, 2064, 16392, WIDE, True, 0),
    ("dx", "bf16", 3001, 520, 1032, WIDE, False, 0), ("dx", "bf16", 3001, 520, 4104, WIDE, False, 0),
    ("dx", "bf16", 600, 4104, 1032, WIDE, True, 0),
    ("dw db", "bf16", 2600, 2568, 2056, WIDE, False, 0), ("dw", "bf16", 3001, 520, 1032, WIDE, True, 0),
    ("db", "bf16", 300, 4104, 4104, WIDE, False, 0), ("dw db dx", "bf16", 2600, 2568, 1032, WIDE, True, 0),
    # ... from padded copies of both operands, of one, of none but the weights' rows
    ("fwd", "bf16", 2611, 2576, 2567, WIDE, False, 2), ("fwd", "bf16", 2600, 2573, 2568, WIDE, False, 0),
    ("fwd", "bf16", 400, 1001, 8195, WIDE, True, 2), ("fwd", "bf16", 400, 1008, 8195, WIDE, True, 2),
    ("fwd", "bf16", 400, 1001, 8192, WIDE, True, 1), ("fwd", "bf16", 300, 2001, 6001, WIDE, True, 2),
    ("dx", "bf16", 700, 1501, 1100, WIDE, True, 2), ("dx", "bf16", 700, 1504, 1100, WIDE, True, 1),
    ("dx", "bf16", 2600, 1301, 1003, WIDE, False, 2), ("dw db", "bf16", 40000, 1031, 129, WIDE, True, 2),
    ("dw", "bf16", 2600, 2571, 2563, WIDE, True, 2), ("db", "bf16", 2600, 2571, 2563, WIDE, True, 1),
    # small batches: 64, 128 and more rows a workgroup, long ranges (whose row tiles begin at different k), many ranges
    ("fwd", "bf16", 33, 8200, 2056, SKINNY, False, 0), ("fwd", "bf16", 64, 8200, 4104, SKINNY, False, 0),
    ("fwd", "bf16", 17, 16392, 4096, SKINNY, True, 0), ("fwd", "bf16", 100, 16392, 2056, SKINNY, False, 0),
    ("fwd", "bf16", 250, 16392, 2056, SKINNY, False, 0), ("fwd", "bf16", 60, 2056, 2056, SKINNY, True, 0),
    ("fwd", "bf16", 3, 8, 100000, SKINNY, True, 0), ("dx", "bf16", 33, 2056, 8200, SKINNY, False, 0),
    ("dx", "bf16", 64, 8200, 4104, SKINNY, True, 0), ("dx", "bf16", 5, 70000, 24, SKINNY, True, 0),
    # few rows: 16 and 32 outputs a workgroup, more weights than 32-bit offsets reach
    ("fwd", "bf16", 9, 1000, 1024, ROWS, False, 0), ("fwd", "bf16", 9, 8200, 1024, ROWS, False, 0),
    ("fwd", "bf16", 4, 8192, 4096, ROWS, False, 0), ("fwd", "bf16", 30, 8200, 520, ROWS, False, 0),
    ("fwd", "bf16", 3, 131080, 8192, ROWS, False, 0), ("fwd", "f32", 8, 8200, 2052, ROWS, False, 0),
    # any size: small and large tiles, K whole and in ranges
    ("fwd", "bf16", 300, 264, 520, TILE, False, 0), ("fwd", "bf16", 90, 77, 4001, TILE, True, 0),
    ("fwd", "bf16", 2100, 2056, 264, TILE, False, 0), ("fwd", "f32", 3, 8, 100000, TILE, True, 0),
    ("fwd", "f32", 1000, 517, 1023, TILE, True, 0), ("fwd", "f32", 2050, 2049, 100, TILE, False, 0),
    ("dx", "bf16", 300, 72, 136, TILE, False, 0), ("dx", "bf16", 90, 4001, 77, TILE, True, 0),
    ("dx", "f32", 5, 70000, 24, TILE, True, 0), ("dx", "f32", 2050, 100, 2049, TILE, False, 0),
    ("dw db", "bf16", 33001, 40, 264, TILE, True, 0), ("dw db", "f32", 40000, 24, 16, TILE, True, 0),
    ("db", "f32", 40000, 24, 16, TILE, True, 0), ("dw db", "f32", 70, 2049, 2050, TILE, False, 0),
    # both backward products in one launch: ranges for both, for one, for none
    ("dw db dx", "bf16", 512, 512, 512, PAIR, False, 0), ("dw db dx", "bf16", 1100, 700, 100, PAIR, True, 0),
    ("dw db dx", "bf16", 700, 1501, 1100, PAIR, True, 0),
    ("dw dx", "f32", 300, 512, 512, PAIR, True, 0), ("db dx", "f32", 1000, 517, 1023, PAIR, True, 0),
    ("dw db dx", "f32", 40, 2000, 33, PAIR, True, 0), ("dw db dx", "f32", 2000, 40, 33, PAIR, True, 0),
    ("dw db dx", "f32", 60, 90, 77, PAIR, False, 0),
]


def _call(which, dtype, B, d_out, d_in, pad):
    t, p = int(dtype == "bf16"), "@4096"
    o, i = d_out + pad, d_in + pad
    if which == "fwd":
        return "linear_fwd", [t, 2, d_out, d_in, B, p, i, p, p, i, "@8192", o, "@1048576", o, t, "@16384", o, p, 1 << 50, None]
    return "linear_bwd", [t, 2, d_out, d_in, B, p, i, p, o, p, i, p if "dw" in which else None, i, p if "db" in which else None, p, i,
                          "@8192", i, "@1048576" if "dx" in which else None, i, t, p, 1 << 50, None]


@pytest.mark.parametrize("pad", [0, 8])
def test_kernels(pad):
    got = launched([_call(*c[:5], pad) for c in CASES])
    wrong = [(c, g) for c, g in zip(CASES, got) if g != c[5]]
    assert not wrong, wrong
