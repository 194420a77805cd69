"""Microscaled 4-bit values on the CPU, from their definition, by whole numbers and exact fractions of 64 bits."""
import numpy as np
import torch

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(v):
    """(codes, scales) of v [rows, cols], in 64 bits that hold fp32 or bf16 values."""
    v = v.double().numpy()
    rows, cols = v.shape
    codes, scales = np.zeros((rows, (cols + 1) // 2), np.uint8), np.zeros((rows, (cols + 31) // 32), np.uint8)
    for r in range(rows):
        for b in range(scales.shape[1]):
            block = v[r, 32 * b:32 * b + 32]
            top = np.abs(block).max()
            if not np.isfinite(top):
                scales[r, b] = 255
                continue
            x = -127 if top == 0 else max(-127, int(np.frexp(top)[1]) - 1 - 2)
            scales[r, b] = x + 127
            t = np.ldexp(np.abs(block), -x)[:, None]
            off = np.abs(t - MAGNITUDES)
            nearest = off.min(1, keepdims=True)
            place = np.where(off == nearest, np.where(np.arange(8) % 2 == 0, 1, 2), 3).argmin(1)   # even places first
            code = place + 8 * np.signbit(block)
            for j, c in enumerate(code):
                codes[r, (32 * b + j) // 2] |= int(c) << (4 * (j % 2))
    return torch.from_numpy(codes), torch.from_numpy(scales)


def values(codes, scales, cols):
    """What they stand for, in 64 bits; codes [..., bytes]."""
    table = torch.from_numpy(np.concatenate((MAGNITUDES, -MAGNITUDES)))
    c = codes.cpu().long()
    v = torch.stack((table[c & 15], table[c >> 4]), -1).flatten(-2)[..., :cols]
    s = torch.from_numpy(np.ldexp(1.0, scales.cpu().numpy().astype(np.int64) - 127))
    s[scales.cpu() == 255] = float("nan")
    return v * s[..., torch.arange(cols) // 32]
