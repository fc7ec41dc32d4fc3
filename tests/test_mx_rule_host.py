"""Which tiles a grouped 4-bit product runs on."""
import pytest

import paper_2605_05049_amd as moe


@pytest.mark.parametrize("experts,rows,n,k,large", [
    # work is rows times columns, also where these do not fill a tile of 256
    (8, 65536, 192, 1024, True), (8, 65536, 192, 512, True), (8, 60000, 96, 1920, True), (64, 24000, 200, 1408, True), (8, 17000, 248, 1024, True),
    (8, 16000, 248, 1024, False), (8, 10000, 504, 1024, True), (8, 8000, 504, 1024, False), (1, 33000, 128, 512, True), (1, 32000, 128, 512, False),
    # ... from 512 k on; below it whole tiles, or three rounds of small tiles
    (8, 60000, 192, 320, False), (8, 65536, 192, 320, True), (8, 65536, 192, 256, True), (8, 10 ** 6, 128, 320, False), (8, 65536, 256, 320, True), (8, 16384, 256, 256, True), (8, 16383, 256, 256, False),
    # mostly empty tiles
    (8, 65536, 64, 1024, False), (8, 2 ** 20, 64, 1920, False), (8, 2 ** 20, 8, 1024, False),
    # whole tiles as before: their work alone, or a long contraction
    (8, 16384, 256, 1024, True), (8, 8192, 512, 1408, True), (8, 8191, 512, 1408, False), (64, 2048, 2048, 1408, True), (64, 512, 2048, 1408, False),
    (8, 2048, 1024, 512, False), (8, 8192, 1024, 512, True), (1000, 16, 2048, 2048, False), (1000, 1024, 2048, 2048, True), (8, 128, 4096, 4096, True),
    # fewer than 8 scales of a row
    (8, 65536, 4096, 224, False),
    # what the call refuses
    (8, 65536, 4100, 512, False),
])
def test_large_tiles(experts, rows, n, k, large):
    assert moe.mxfp4_grouped_gemm_large_tiles(experts, rows, n, k) is large
