"""The 8-bit rows' largest numbers: what is finite in bf16 stays so."""

import numpy as np
import torch

from oracle import paged


def test_a_finite_number_stays_finite():
    bits = torch.arange(0x7e00, 0x7f80, dtype=torch.int16).view(torch.bfloat16).double().numpy()
    x = np.zeros((2 * bits.size, 8))
    x[:, 3] = np.concatenate([bits, -bits])
    codes, e = paged.encode(x)
    back = torch.from_numpy(paged.decode(codes, e)).to(torch.bfloat16).double().numpy()
    assert np.isfinite(back).all()
    assert (np.abs(back[:, 3] - x[:, 3]) <= 2.0 ** -4 * np.abs(x[:, 3])).all()
    # only the numbers whose nearest code is 256 or more are held back
    held = np.abs(x[:, 3]) >= 248.0 * 2.0 ** 120
    assert held.sum() == 16 and (np.abs(back[held, 3]) == 240.0 * 2.0 ** 120).all()
    y = torch.from_numpy(x[:, 3] / 2.0 ** e.astype(float)).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(codes[~held, 3], y[~held])
