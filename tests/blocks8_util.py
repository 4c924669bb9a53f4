"""Tensors in 8 bits written out in 64 bits: the definition of include/co3.h, for the tests."""
import numpy as np
import torch

# the 256 numbers of e4m3: a sign, four bits of an exponent, three of a fraction; both codes of 127 are NaN
NUMBERS = torch.tensor([(-1.0 if v & 128 else 1.0) * (float("nan") if v & 127 == 127 else
                                                      (v & 7) * 2.0 ** -9 if not v & 120 else (8 + (v & 7)) * 2.0 ** ((v >> 3 & 15) - 10))
                        for v in range(256)], dtype=torch.float64)


def numbers(values, scales, cols, block_rows):
    """float64 [batch, rows, cols] of values [batch, rows, ld] and scales [batch, columns of blocks, ...]."""
    v = NUMBERS.to(values.device)[values[:, :, :cols].long()]
    row = torch.arange(v.shape[1], device=v.device) // block_rows
    col = torch.arange(cols, device=v.device) // 128
    e = scales.double() - 127
    return v * torch.exp2(e.cpu()).to(v.device)[:, col][:, :, row].mT


def stored(x, block_rows):
    """(values uint8 [batch, rows, up16(cols)], scales uint8) of float64 x, block by block, in NumPy; what is between is 0."""
    x = x.cpu().numpy()
    batch, rows, cols = x.shape
    n, c = -(-rows // block_rows), -(-cols // 128)
    values = np.zeros((batch, rows, -(-cols // 16) * 16), np.uint8)
    scales = np.zeros((batch, c, -(-n // 16) * 16), np.uint8)
    grid = NUMBERS[:127].numpy()          # rising; code = place
    for b in range(batch):
        for i in range(n):
            for j in range(c):
                t = x[b, i * block_rows:(i + 1) * block_rows, j * 128:(j + 1) * 128]
                fine = np.isfinite(t)
                most = np.abs(t[fine]).max() if fine.any() else 0.0
                e = -126
                if most == 0:
                    e = 0
                else:
                    while most > 448.0 * 2.0 ** e:
                        e += 1
                scales[b, j, i] = e + 127
                a = np.where(fine, np.abs(t), 0) * 2.0 ** -e
                code = np.clip(np.searchsorted(grid, a), 1, 126)      # the number at or above, and the one below it
                up, down = grid[code] - a, a - grid[code - 1]
                code = np.where((down < up) | ((down == up) & ((code - 1) % 2 == 0)), code - 1, code)
                code = np.where(np.signbit(t), code + 128, code)
                values[b, i * block_rows:(i + 1) * block_rows, j * 128:min(cols, (j + 1) * 128)] = np.where(fine, code, 127)
    return values, scales
