"""Sizes (rows, columns, output channels) of the linear layers' tests. Between them they reach every kind of product: few rows
in one launch, tiles of 64, 128 and 256, whole and in parts, and 8-bit rows taken as they are."""

SIZES = [(2000, 1003, 771), (2500, 520, 4100), (4097, 4099, 136), (300, 5000, 640), (20_001, 256, 128), (1, 9000, 4096),
         (3, 70, 9000), (9000, 70, 3), (513, 2049, 2100), (50_001, 8, 8), (8, 50_001, 16), (5000, 3001, 1500),
         (8192, 4100, 264), (1000, 1000, 9000), (2000, 2000, 5000), (4097, 4099, 2100)]
