"""Shapes whose product with 4-bit weights is that of values laid out in the type (csrc/slz_i4_route.h), for any group and for 16-bit and f32 inputs alike.
tests/test_clear_cpu_i4_laid_out.py holds them against the choice itself and tests/test_gpu_clear_i4_laid_out.py runs them."""

# (m, n, k): a row of less than eight entries, whole blocks, ends inside blocks, groups and tiles
SHAPES = [(60, 40, 5), (2048, 2048, 128), (2003, 2050, 167), (2500, 2300, 200)]
