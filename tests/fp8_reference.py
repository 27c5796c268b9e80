"""Plain 64-bit forms of the 8-bit matrices in include/chgnet_ops.h and of their products. Test infrastructure; shares no code
with the library."""
import math

import torch

U = 2.0 ** -24


def quantize(x, block_rows=1):
    """(codes as e4m3 values in 64 bits [rows, cols], exponent bytes [rows / block_rows, cols / 128]) of x (CPU)."""
    rows, cols = x.shape
    x = x.double()
    nr, nb = -(-rows // block_rows), -(-cols // 128)
    q, byte = torch.zeros(rows, cols, dtype=torch.float64), torch.zeros(nr, nb, dtype=torch.int64)
    for i in range(nr):
        for j in range(nb):
            b = x[i * block_rows:(i + 1) * block_rows, j * 128:(j + 1) * 128]
            if not bool(torch.isfinite(b).all()):
                byte[i, j] = 255
                continue
            big = float(b.abs().max())
            e = -126
            if big > 0:
                m, k = math.frexp(big)  # big = m 2^k, 1/2 <= m < 1; 448 = 0.875 2^9
                e = max(-126, k - 9 + (m > 0.875))
            byte[i, j] = e + 127
            v = b * 2.0 ** -e
            _, k = torch.frexp(v)
            step = torch.ldexp(torch.ones_like(v), (k - 1).clamp(min=-6) - 3)  # three bits behind the leading one
            q[i * block_rows:(i + 1) * block_rows, j * 128:(j + 1) * 128] = torch.round(v / step) * step
    return q, byte


def values(q, byte, block_rows=1):
    s = torch.where(byte == 255, float("nan"), torch.ldexp(torch.ones(byte.shape, dtype=torch.float64), byte - 127))
    return q * s.repeat_interleave(block_rows, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]


def product(a, b, dtype=torch.float32):
    """a b^T in 64 bits, and a bound of the sum before its rounding to dtype. Products of two codes are exact. fp32: as if each
    of an instruction's 128 products were added on its own and the sum cut off each time (2 U), then the instructions' results
    and those of the parts of K. 16 bits: besides, each of eight products is cut off at 2^-13 of the power of two of the
    largest, so eight of them lose at most 8 2^-13 of that one, and all at most 2^-10 of the sum of all magnitudes."""
    K = a.shape[1]
    whole = a.abs() @ b.abs().T
    return a @ b.T, ((2 * min(K, 128) + 2 * math.ceil(K / 128) + 40) * U + (2.0 ** -10 if dtype != torch.float32 else 0)) * whole + 1e-37
