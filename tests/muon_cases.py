"""Lists of matrices that reach every form of the orthogonalised update: which kernels, and how many chunks of 32 columns a wavefront
works through (a block's wavefronts take 32 columns of X each at a time)."""

# name -> (tiles of 32 rows, one launch, blocks add their shares by themselves, chunks of a wavefront), the matrices
FORMS = {
    "alone1": ((1, True, True, None), [(32, 768), (700, 20), (1, 1)]),
    "alone2": ((2, True, True, None), [(40, 380), (384, 33), (64, 64)]),
    "direct1": ((1, False, True, 1), [(20, 1100), (3000, 32), (9, 40)]),
    "direct2": ((2, False, True, 1), [(44, 700), (2000, 40), (5, 5)]),
    "sums1": ((1, False, False, 1), [(8, 12300), (40, 9)]),
    "sums2": ((2, False, False, 1), [(36, 4100), (60, 50)]),
    "sums4": ((4, False, False, 1), [(80, 90), (700, 128), (3, 5)]),
    # wavefronts with several chunks one after the other; last blocks with fewer, and wavefronts with fewer than their neighbours
    "direct1_two": ((1, False, True, 2), [(32, 24576), (24570, 31), (20, 24000), (5, 60)]),
    "direct2_two": ((2, False, True, 2), [(64, 8192)] * 5 + [(8190, 40)] * 4 + [(70, 33)]),
    "sums1_two": ((1, False, False, 2), [(16, 50000), (20011, 32), (60, 5)]),
    "sums2_two": ((2, False, False, 2), [(64, 40000), (30011, 60), (50, 70)]),
    "sums4_two": ((4, False, False, 2), [(128, 22016), (11007, 127), (688, 128), (70, 100)]),
    "sums4_three": ((4, False, False, 3), [(128, 22016), (22005, 100), (65, 22000), (700, 128)]),
    "sums1_many": ((1, False, False, 33), [(2, 2 ** 21), (65, 3), (3, 1000)]),
}


def chunks(shape):
    return -(-max(shape) // 32)
