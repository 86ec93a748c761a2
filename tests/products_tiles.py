"""Sizes at which a product takes a certain shape of tile (rows of X, rows of W): which one is asserted on the host, the results on the device."""
import numpy as np

# Few rows and long K, 9 to 57 blocks of 128 columns, the last one of 16: every wave has blocks, some of them one more than others.  (shape, m, n, k)
DENSE = [((16, 64), 16, 14336, 4096), ((16, 64), 12, 14336, 1040), ((16, 64), 11, 20001, 2064), ((16, 32), 16, 8000, 2448), ((16, 32), 5, 9001, 2064), ((16, 32), 14, 9001, 4240),
         ((16, 32), 7, 6001, 1040), ((16, 16), 8, 3000, 7184),
         # several tiles to a workgroup
         ((128, 128), 4171, 3934, 592), ((128, 128), 4137, 3924, 1040), ((128, 128), 4205, 3876, 2064)]

# (shape, rows of each expert, n, k)
FEW = [((16, 64), [2, 0, 4], 9001, 2064), ((16, 64), [2, 2, 2], 9001, 2064), ((16, 64), [2, 1, 0], 12000, 4112), ((16, 64), [2, 2, 1, 0, 3, 1, 1, 2, 2, 1, 3, 2], 6000, 1040),
       ((16, 64), [1] * 8, 9001, 2064), ((64, 128), [1] * 8, 4000, 7168), ((64, 256), [1] * 15, 4000, 7168), ((64, 128), [2, 0, 1, 3, 1, 1, 0, 7], 4000, 7184), ((64, 256), [1, 2, 0, 2, 1, 2], 9001, 4112)]

# (shape, rows, experts, how unlike their numbers of rows are, n, k): several tiles to a workgroup, K from fewer blocks than the ring has buffers up
MANY = [((64, 128), 1896, 126, 0.5, 1037, 4640), ((64, 128), 900, 79, 0.3, 2360, 2960), ((64, 128), 1400, 111, 1.0, 1611, 2064), ((64, 128), 20000, 600, 0.5, 104, 1168),
        ((128, 128), 11529, 3, 0.2, 517, 1040), ((128, 128), 9694, 158, 0.5, 1028, 2064), ((128, 128), 5483, 154, 0.5, 1066, 400), ((128, 128), 4587, 195, 0.3, 886, 272),
        ((128, 128), 9845, 71, 0.7, 1600, 1040)]


def counts_of(rows, experts, unlike):
    """Rows of each expert, seven less than there are in all."""
    rng = np.random.default_rng(rows)
    share = np.exp(rng.normal(0, unlike, experts))
    return rng.multinomial(rows - 7, share / share.sum()).tolist()


def tiles(shape, counts, n):
    return sum(-(-c // shape[0]) for c in counts) * -(-n // shape[1])
