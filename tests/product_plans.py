"""Sizes (rows, columns, output channels) of the linear layers' tests. SIZES reach between them every kind of
product: few rows in one launch, float32 as it is, tiles of 64, 128 and 256, whole and in parts, and 8-bit rows taken as they
are. FEW are on both sides of the numbers of rows that choose between the kernels of few rows, of tiles, pieces and steps."""

SIZES = [(2000, 1003, 771), (2500, 520, 4100), (4097, 4099, 136), (300, 5000, 640), (20_001, 256, 128), (1, 9000, 4096),
         (3, 70, 9000), (9000, 70, 3), (513, 2049, 2100), (50_001, 8, 8), (8, 50_001, 16), (5000, 3001, 1500),
         (8192, 4100, 264), (1000, 1000, 9000), (2000, 2000, 5000), (4097, 4099, 2100), (100, 70, 9000), (400, 900, 700)]

FEW = [(rows, cols, n) for rows in (1, 2, 16, 17, 32, 33, 64, 65, 384, 385)
       for cols, n in ((1, 1), (3, 5), (7, 300), (64, 16), (129, 33), (260, 31), (1030, 70), (257, 8300), (2050, 4100))]
