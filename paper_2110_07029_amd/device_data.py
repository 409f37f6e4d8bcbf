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


class _Is(dict):
    """Whether one of torch's element types is among the named."""

    def __init__(self, *names):
        self.names = names

    def __missing__(self, dtype):
        self[dtype] = str(dtype) in self.names
        return self[dtype]


_TYPES = _Types()
_FLOAT = _Is("torch.float32")
_WORD = _Is("torch.int32", "torch.uint32")
_LIST = ctypes.POINTER(asgd_csr)
_ANY = 1 << 31  # more rows or columns than any matrix has


def matrix(t) -> asgd_matrix:
    """A 2-d tensor (unit stride along a row) as an asgd_matrix; the tensor must outlive its use."""
    shape = t.shape
    if len(shape) != 2:
        raise ValueError("a matrix has two dimensions")
    rows, cols = shape
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
    [words] for one mask for all rows) and asgd_csr lists.  Other types and strides raise ValueError, as
    do tensors too short for the logits where the rules meet them.  The tensors must outlive the rules' use."""
    at = mask = None
    ld, rows, cols = 0, _ANY, _ANY
    if bias is not None:
        if bias.stride() != (1,) and (bias.dim() != 1 or bias.numel() > 1) or not _FLOAT[bias.dtype]:
            raise ValueError("rules.bias is a contiguous float32 tensor of one dimension")
        at, cols = bias.data_ptr(), bias.numel()
    if allowed is not None:
        shape, step = allowed.shape, allowed.stride()
        if len(shape) not in (1, 2) or (step[-1] != 1 and shape[-1] > 1) or not _WORD[allowed.dtype]:
            raise ValueError("rules.allowed holds int32 or uint32 words, [rows, words] or [words], with unit stride along a row")
        mask, cols = allowed.data_ptr(), min(cols, 32 * shape[-1])
        if len(shape) == 2:
            rows = shape[0]
            ld = step[0] if rows > 1 else shape[1]
    r = asgd_logit_rules(at, mask, ld, None if seen is None else _LIST(seen), None if row_bias is None else _LIST(row_bias),
                         repetition, frequency, presence)
    if cols != _ANY:
        r.covers = rows, cols
    return r
