"""Sizes (tokens, channels, columns) of int8 products, by the kernel that makes them: its tiles, tokens by channels.
Shared by the GPU tests of the results and the CPU test that these sizes do choose these kernels."""

# ragged in tokens and channels, an odd and an even number of 128-column steps, one step, one token past whole tiles
SIZES = {
    "16 x 16 split": [(1, 1, 1), (3, 5000, 700), (250, 255, 1100), (2000, 7, 129)],
    "32 x 16 split": [(300, 321, 2000), (33, 1999, 130), (511, 250, 500)],
    "32 x 32 split": [(500, 509, 1000), (997, 250, 100), (33, 4999, 513)],
    "64 x 64": [(65, 4001, 4000), (1771, 1003, 771), (129, 5000, 60), (10_001, 801, 800), (65_537, 127, 1000)],
    "128 x 128": [(2041, 2047, 2000), (2001, 3999, 1900), (65_409, 127, 1000), (4090, 4083, 900)],
    "256 x 256": [(4081, 4079, 4000), (3841, 4095, 3900), (4095, 3842, 4100), (7937, 4001, 2500),
                  (8161, 8177, 2600), (5793, 2801, 4000)],
}
KERNELS = list(SIZES)  # in the order of the library's numbers
