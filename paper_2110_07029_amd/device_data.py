"""Device-resident CSR datasets whose batches are zero-copy row slices, and torch
tensors as the library's dense arguments.

The whole synthetic dataset is staged once in HBM (torch tensors are used only
as device memory); a batch handed to the library is a pointer into the
dataset's indptr plus the host's nnz count for that slice.
"""
from __future__ import annotations

import ctypes

import numpy as np

from ._binding import ASGD_BF16, ASGD_F16, ASGD_F32, asgd_csr, asgd_fp4, asgd_logit_rules, asgd_matrix


class DeviceCSR:
    def __init__(self, csr, device="cuda"):
        import torch
        indptr = np.asarray(csr.indptr, np.int64)
        if indptr[-1] >= 2 ** 31:
            raise ValueError("dataset has more than 2^31 entries")
        self.indptr_host = indptr
        self.n_cols = int(csr.n_cols)
        self.n_rows = len(indptr) - 1
        self.indptr = torch.from_numpy(indptr.astype(np.int32)).to(device)
        self.indices = torch.from_numpy(np.asarray(csr.indices, np.int32)).to(device)
        self.values = None if csr.values is None else torch.from_numpy(
            np.asarray(csr.values, np.float32)).to(device)

    def batch(self, r0: int, r1: int) -> asgd_csr:
        """Rows [r0, r1) as an asgd_csr (indptr offsets stay absolute)."""
        if not (0 <= r0 < r1 <= self.n_rows):
            raise ValueError("row range out of bounds")
        nnz = int(self.indptr_host[r1] - self.indptr_host[r0])
        return asgd_csr(r1 - r0, self.n_cols, nnz, self.indptr.data_ptr() + 4 * r0,
                        self.indices.data_ptr(),
                        None if self.values is None else self.values.data_ptr())

    def nnz(self, r0: int, r1: int) -> int:
        return int(self.indptr_host[r1] - self.indptr_host[r0])


class _Types(dict):
    """torch's element types as the library's, looked up without importing torch before it is needed."""

    def __missing__(self, dtype):
        code = {"torch.float32": ASGD_F32, "torch.bfloat16": ASGD_BF16, "torch.float16": ASGD_F16}.get(str(dtype))
        if code is None:
            raise ValueError(f"no matrix of {dtype}")
        self[dtype] = code
        return code


_TYPES = _Types()


def matrix(t) -> asgd_matrix:
    """A 2-d tensor (unit stride along a row) as an asgd_matrix; the tensor must outlive its use."""
    if t.dim() != 2:
        raise ValueError("a matrix has two dimensions")
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("a matrix needs unit stride along a row")
    return asgd_matrix(rows, cols, ld if rows > 1 else cols, _TYPES[t.dtype], t.data_ptr())


def fp4_matrix(codes, scales) -> asgd_fp4:
    """uint8 tensors, codes [rows, cols / 2] and scales [rows, cols / 32], as an asgd_fp4."""
    rows, half = codes.shape
    if codes.element_size() != 1 or scales.element_size() != 1 or half % 16:
        raise ValueError("codes and scales are bytes, codes with a multiple of 16 columns")
    if tuple(scales.shape) != (rows, half // 16) or not (codes.is_contiguous() and scales.is_contiguous()):
        raise ValueError("codes [rows, cols / 2] and scales [rows, cols / 32] must be contiguous")
    return asgd_fp4(rows, 2 * half, codes.data_ptr(), scales.data_ptr())


def logit_rules(bias=None, allowed=None, seen=None, repetition: float = 1.0, frequency: float = 0.0,
                presence: float = 0.0, row_bias=None) -> asgd_logit_rules:
    """Rules from tensors (bias: float32 [L]; allowed: int32 / uint32 words, [rows, words] or
    [words] for one mask for all rows) and asgd_csr lists."""
    ld = 0 if allowed is None or allowed.dim() == 1 else allowed.stride(0) if allowed.shape[0] > 1 else allowed.shape[1]
    r = asgd_logit_rules(None if bias is None else bias.data_ptr(), None if allowed is None else allowed.data_ptr(), ld,
                         None, None, repetition, frequency, presence)
    if seen is not None:
        r.seen = ctypes.pointer(seen)
    if row_bias is not None:
        r.row_bias = ctypes.pointer(row_bias)
    return r
