"""Sizes of the tests that hold whole tensors of the layers to close bounds, on the GPU and, the bounds themselves, on the CPU."""
SMS = 148

# fp32, sums of up to 192 terms each way: three tiles of rows and of columns, whole and ragged, one with a row more than the kernels of a few rows take
FP32_SIZES = [(128, 64, 96), (192, 128, 128), (160, 192, 192), (97, 61, 131), (40, 30, 77), (17, 190, 100)]

# (rows, K, N, terms of the sums that are long); narrow tiles with two buffers for a run's sums, and so many wide ones that they have one
LONG = [(300, 16384, 96, 16384), (4096, 16384, 1024, 16384)]

# the one-pass kernel: so many tiles of 128 rows a block, and a few rows less
SMALL_ROWS = [tiles * SMS * 128 - 1000 for tiles in (1, 4, 5, 8, 9, 13)]
SMALL_SIZES = [(64, 64), (64, 192), (128, 128), (48, 96), (192, 64), (72, 136)]
# the three kernels, ragged sizes among them
MANY_ROWS = [(20000, 64, 128), (40013, 48, 64), (5000, 192, 64), (3001, 320, 640), (70000, 16, 16), (9000, 100, 36), (113664, 64, 128), (30011, 320, 72)]
NORM_ROWS = [(5000, 64), (20011, 48), (3001, 777), (200000, 64), (9001, 1024), (2500, 5001)]

# Gradients that are sums over rows, fp32: a run's 32 steps of 2 u, u for each of 64 runs in a part and 32 + 592 / 32 parts, 8 u and less for a slope or
# a normed value: below 256 u.  With a rounding of g to bf16, at random and 2^-8 at most, that alone.
GRAD_SUMS, GRAD_H = 2.0 ** -16, 2.0 ** -8 + 2.0 ** -16
