"""Sizes of products that reach every kernel of jenga_matmul: (m, n, k, type of the result) by (rows without tiles, tile, LDS tiles).

Of the kernels with tiles, the first size has no more tiles than workgroups, partial ones at both ends among them; the others have several
for each workgroup: whole tiles in front of partial ones (the stores of a whole tile are still under way when the next one's copies are
waited for), and whole tiles alone.  k: numbers of blocks of 128 that are no multiple of the LDS tiles or of four, the last one partly filled."""

ROWS_16, ROWS_32 = (16, 0, 0, 0), (32, 0, 0, 0)
TILES_256, TILES_64, TILES_128_DEEP, TILES_128 = (0, 256, 256, 2), (0, 64, 128, 4), (0, 128, 128, 4), (0, 128, 128, 2)

SIZES = {
    ROWS_16: [(7, 1030, 900)],
    ROWS_32: [(27, 700, 1300)],
    TILES_64: [(200, 1000, 700), (64, 128, 2000)],
    TILES_128_DEEP: [(1000, 2100, 600), (1024, 2176, 1152)],
    TILES_128: [(2300, 2400, 300), (4500, 5200, 384), (4096, 5120, 896)],
    TILES_256: [(3900, 2500, 600), (5200, 5300, 384), (5120, 5632, 896)],
}
CASES = [(kernel, m, n, k, out) for kernel, sizes in SIZES.items() for m, n, k in sizes for out in ("bf16", "f16", "f32")
         if not (kernel == TILES_256 and out == "f32")]
