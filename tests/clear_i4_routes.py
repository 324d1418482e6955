"""Shapes that take each kernel of a product with 4-bit weights (csrc/slz_i4_route.h), with ends inside blocks, groups and tiles.  tests/test_clear_cpu_i4_routes.py holds them against
the choice itself and tests/test_gpu_clear_i4_routes.py runs them."""

# (m, n, k, group), f32, (kernel, kind)
ROUTES = [
    ((1, 45, 3, 32), False, ("thin", 0)),
    ((2, 9001, 1290, 64), False, ("thin", 0)),         # 32 rows of weights a workgroup
    ((8, 4001, 500, 128), False, ("thin", 0)),
    ((3, 100, 9000, 32), False, ("thin", 0)),          # more scales and entries than are under way at once
    ((8, 500, 6007, 64), False, ("thin", 0)),          # more shared memory than 64 KiB
    ((2, 300, 9001, 128), True, ("thin", 0)),
    ((5, 700, 1000, 64), True, ("thin", 0)),
    ((2, 8300, 260, 128), True, ("thin", 0)),
    ((13, 1000, 2100, 128), False, ("rows", 0)),
    ((9, 333, 8, 32), False, ("rows", 1)),
    ((40, 600, 1555, 64), False, ("rows", 0)),
    ((11, 17000, 300, 64), False, ("rows", 1)),
    ((1, 33000, 129, 32), False, ("rows", 1)),
    ((90, 5000, 1100, 32), False, ("rows", 2)),
    ((200, 3001, 700, 128), False, ("rows", 2)),
    ((300, 3500, 1290, 64), False, ("rows", 2)),
    ((250, 4090, 2053, 32), False, ("rows", 3)),
    ((70, 16400, 517, 128), False, ("rows", 2)),
    ((500, 8100, 700, 64), False, ("rows", 4)),
    ((250, 16001, 2053, 32), False, ("rows", 4)),
    ((1000, 4001, 1111, 128), False, ("rows", 4)),
    ((9, 5001, 777, 32), True, ("rows", 0)),
    ((100, 1000, 1030, 64), True, ("rows", 0)),
    ((33, 70, 9001, 128), True, ("rows", 0)),
    ((3000, 4000, 300, 64), False, ("tiles", 0)),
    ((2500, 3100, 777, 32), False, ("tiles", 0)),
    ((40, 300, 7, 128), False, ("tiles", 0)),
    ((4000, 2300, 500, 128), True, ("tiles", 0)),
    ((60, 40, 5, 32), True, ("tiles", 0)),
]
