"""Rows of logits for the GPU tests, and how far results in 32 or fewer bits may be from 64-bit ones."""
import numpy as np
import torch

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}      # relative rounding of a value
SMALLEST = {"fp32": 2.0 ** -126, "bf16": 2.0 ** -126, "fp16": 2.0 ** -25}    # absolute: half of fp16's smallest step, flushed results of fp32


def place(z, dtype, pad=0, offset=0):
    """The rows of numpy matrix z on the GPU, rounded to dtype, every row followed by `pad` NaN and the whole preceded by `offset`
    NaN, so that rows start at other alignments and a read outside a row shows.  Returns the strided view and its
    values in 64 bits."""
    rows, V = z.shape
    buf = torch.full((offset + rows * (V + pad) + 16,), float("nan"), dtype=DTYPES[dtype], device="cuda")
    view = buf[offset:offset + rows * (V + pad)].view(rows, V + pad)[:, :V]
    view.copy_(torch.from_numpy(np.ascontiguousarray(z)).to(DTYPES[dtype]))
    return view, view.double().cpu().numpy()


def sum_error(V):
    """Bound on the relative error of a row's fp32 sum of exp((z - m) * c): every term's exponent t carries three
    roundings (the difference, the factor c, the product), 3 * 2^-24 * |t| * ln 2 with the terms' weighted mean of |t| at
    most log2 V, and two units of the exponential; a thread adds at most V/64 terms one after the other, each addition
    and each rescaling of what was added one rounding, then fewer than 64 more across threads."""
    return 2.0 ** -24 * (3 * np.log(2) * np.log2(max(V, 2)) + 4 + 2 * (V / 64) + 64)
