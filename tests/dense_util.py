"""Matrices in larger arrays for the tests of dense layers and layer norm: rows of any pitch at any element, and a check that
nothing around a result was written."""
import numpy as np
import torch

DEV = "cuda:0"
TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}
# half a step of each type, relative
HALF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
MARK = 0x4D4D  # a bit pattern of both types, finite


def pitch8(n):
    return n if n == 1 else (n + 7) // 8 * 8


class Matrix:
    """[rows][cols] at a pitch, `offset` elements into an array whose other elements are `fill`."""

    def __init__(self, rows, cols, dtype, ld=None, offset=0, values=None, fill=float("nan"), device=DEV):
        self.rows, self.cols, self.ld, self.offset = rows, cols, pitch8(cols) if ld is None else ld, offset
        self.kind = TORCH.get(dtype, dtype)
        n = offset + (rows - 1) * self.ld + max(self.ld, (cols + 7) // 8 * 8) + 64
        self.whole = torch.full((n,), fill, dtype=self.kind, device=device)
        if values is not None:
            self.view.copy_(torch.as_tensor(values, device=device).to(self.kind))

    @property
    def view(self):
        return self.whole[self.offset:].as_strided((self.rows, self.cols), (self.ld, 1))

    @property
    def data(self):
        return self.whole[self.offset:]

    def f64(self):
        return self.view.double().cpu().numpy()

    def surroundings(self):
        """Bits of everything beside the matrix."""
        bits = self.whole.clone().view(torch.int32 if self.kind is torch.float32 else torch.int16)
        bits[self.offset:].as_strided((self.rows, self.cols), (self.ld, 1)).zero_()
        return bits


def result(rows, cols, dtype, ld=None, offset=0):
    return Matrix(rows, cols, dtype, ld, offset, fill=77.0)


def workspace(nbytes):
    """Poisoned: nothing may be taken from what a workspace held before."""
    return torch.full((max(nbytes, 1),), 0xFF, dtype=torch.uint8, device=DEV), nbytes


def integers(rng, rows, cols, most=2):
    return rng.integers(-most, most + 1, (rows, cols)).astype(np.float64)


def rounded(v, dtype):
    """Values (exact in float32) in the type, nearest even."""
    return torch.as_tensor(np.asarray(v, dtype=np.float32)).to(TORCH[dtype]).double().numpy()
