"""Shared by the tests of every form of the dense layers' products, pinned by the switches LUTNN_DENSE_FORM and LUTNN_DENSE_SPLITS."""
import torch

import dense_util as du

# tile sizes by form; those that read their operands as they are lay nothing out
TILES = {"256x256": (256, 256), "128x256": (128, 256), "128x128": (128, 128), "64x128": (64, 128), "64x64": (64, 64), "32x64": (32, 64),
         "64x64 as is": (64, 64), "32x64 as is": (32, 64), "32x32 as is": (32, 32)}
FORMS = {"f32": ("memory", "128x256", "128x128", "64x64 as is", "32x32 as is"),
         "bf16": ("256x256", "128x128", "64x128", "64x64", "32x64", "64x64 as is", "32x64 as is")}
FORMS["f16"] = FORMS["bf16"]

# A single product of fp32 values from three bf16 parts each, a = h + m + l.  Parts are cut, so that m is less than 2^-7 of a and l less
# than 2^-15, and what the six products leave out, m l' + l m' + l l', less than 2^-21 (1 + 2^-8) = 8.04 u.  Six additions, each off by at
# most 2 u of the sum, where the matrix instructions cut.
ONE_TERM = 22 * du.U


def one_per_row(rows, cols, seed):
    """An fp32 matrix with one value in every row, at columns that go round all of them, and where it is."""
    at = (torch.arange(rows) * 7 + cols - 1) % cols
    A = torch.zeros((rows, cols))
    A[torch.arange(rows), at] = torch.randn(rows, generator=torch.Generator().manual_seed(seed)) + 0.1
    return A.cuda(), at.cuda()


def check_relative(got, want, share):
    du.check(got, want, share * want.abs() + du.smallest(torch.float32))
