"""The workspace of split tiles holds the parts that there are (no GPU needed).

64 fp32 matrices of 200 x 1000: each has 200 columns of X X^T in tiles of 256 x 128 (or twice as
many of half the width), 16 stages deep, in two parts of fp32 sums.  A matrix's iterates are four buffers of 200 x 1024 fp16 and four of 200 x 256; the
tables (a few kilobytes: tensor maps, tiles, units) and everything else are below 16 KB each."""


def test_parts_take_their_own_sums_and_no_more(lib):
    n = 64
    arr = (lib.zo_muon_matrix * n)(*[
        lib.zo_muon_matrix(0x1000, 0x2000, 0x3000, 200, 1000, 1000, 1000, 0, 0) for _ in range(n)])
    iterates = 4 * 2 * 200 * 1024 + 4 * 2 * 200 * 256
    parts = 2 * 2 * 4 * 256 * 128
    need = lib.LIB.zo_muon_workspace(arr, n)
    assert n * (iterates + parts) < need < n * (iterates + parts + (16 << 10)) + (1 << 20)
