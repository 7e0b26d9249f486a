"""Inputs and guarded buffers for the tests of the steps around the linears."""
import numpy as np
import torch

from paper_2510_27527_b200 import synth

GUARD = {torch.bfloat16: -77.0, torch.float32: -77.0}


def guarded(rows, cols, dtype, extra_cols=8, extra_rows=3):
    """(view [rows, cols], whole buffer): a matrix inside a larger one that a call must leave as it is."""
    ld = (cols + 7) // 8 * 8 + extra_cols
    buf = torch.full((rows + extra_rows, ld), GUARD[dtype], dtype=dtype, device="cuda")
    return buf[:rows, :cols], buf


def untouched(view, buf):
    rows, cols = view.shape
    return bool((buf[rows:] == GUARD[buf.dtype]).all()) and bool((buf[:, cols:] == GUARD[buf.dtype]).all())


def device_rows(x: np.ndarray, dtype, extra_cols=8):
    """A float32 host matrix on the device, in a buffer whose other elements are NaN: reading them would show."""
    rows, cols = x.shape
    buf = torch.full((rows, (cols + 7) // 8 * 8 + extra_cols), float("nan"), dtype=dtype, device="cuda")
    buf[:, :cols] = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()
    return buf[:, :cols]


def host(t: torch.Tensor) -> np.ndarray:
    return t.detach().double().cpu().numpy()


def inputs(rows, cols, seed, dtype=torch.bfloat16, scale=1.0, hot=True):
    x, _ = synth.activations(rows, cols, seed, n_outlier=max(1, cols // 50) if hot else 0, factor=30.0)
    if dtype == torch.float32:  # more bits than BF16 has
        x = x * (1 + np.random.default_rng(seed).random(x.shape, dtype=np.float32) * np.float32(0.01))
    return (x * np.float32(scale)).astype(np.float32)


BF16 = 2.0 ** -8  # half a step of a rounding to BF16, relative
F32 = 2.0 ** -24
