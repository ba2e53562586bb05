"""Inputs of the serving tests, and their device tensors."""
from __future__ import annotations

import numpy as np
import torch

from oracle import serving_oracle as so

HALF_STEP = 2.0 ** -8           # of a bf16 rounding, relative to the value
# fp32 evaluation of a rotation, relative to the pair: the reduced angle in turns is off by 2^-25, so by 2^-25 * 2 pi = 1.9e-7
# in radians; cos and sin by 2 units (2.4e-7); two products and a sum by 3 * 2^-24 = 1.8e-7; a magnitude by 6e-8
TURN = 1.0e-6


def bf16(x: np.ndarray) -> np.ndarray:
    """Rounded to bf16, in fp64."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).double().numpy()


def to_device(x: np.ndarray) -> torch.Tensor:
    """fp64 holding bf16 values -> bf16 on the device."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


def e4m3_to_device(x: np.ndarray) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.float8_e4m3fn).cuda()


def ints(x) -> torch.Tensor:
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def host(t: torch.Tensor) -> np.ndarray:
    return t.float().cpu().numpy().astype(np.float64)


def bits(t: torch.Tensor) -> np.ndarray:
    return t.contiguous().view(torch.uint8).cpu().numpy()


def layout_of(x: torch.Tensor, how: str) -> torch.Tensor:
    """The same values [heads, tokens, d] as a view with other strides: "dense", "fused" (heads inside one projection
    with others behind them), "gaps" (rows apart by more than d)."""
    h, t, d = x.shape
    if how == "dense":
        return x.contiguous()
    if how == "fused":
        wide = torch.full((t, h + 3, d), float("nan"), dtype=x.dtype, device=x.device)
        view = wide[:, 1:1 + h].transpose(0, 1)
    else:
        wide = torch.full((h, t + 2, d + 24), float("nan"), dtype=x.dtype, device=x.device)
        view = wide[:, 1:1 + t, 8:8 + d]
    view.copy_(x)
    return view


def make_table(rng, lengths, page, spare=2, wider=1):
    """Pages of the sequences in no order; -1 behind each sequence's last one."""
    counts = [-(-max(n, 0) // page) for n in lengths]
    n_pages = max(sum(counts) + spare, 1)
    order = rng.permutation(n_pages)
    table = np.full((len(lengths), max(max(counts), 1) + wider), -1, dtype=np.int64)
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = order[at:at + c]
        at += c
    return table, n_pages


def check_bf16(got, ref, slack, what=""):
    """|got - ref| within half a step of ref and what the arithmetic in front of the rounding may be off (with its own share
    of a step)."""
    bound = HALF_STEP * (np.abs(ref) + slack) + slack + 1e-37
    err = np.abs(got - ref)
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(err / bound):.3g} of the bound at {np.argwhere(bad)[0]}"


def check_attention(got_out, got_lse, q, k_values, v_values, lengths, cu, table, window, sinks, scale=None, v_rel=0.0):
    """Outputs against the oracle.  A probability is off by its score's error twice (own score and the sum), by the
    exponential's and by one rounding to bf16; a score of d products summed in fp32 by d * 2^-24 of scale * sum |q||k|,
    and by 4 roundings of scale and differences of the scaled score; v_rel: further roundings of P v."""
    d = q.shape[2]
    out, lse, spread, reach = so.attention(q, k_values, v_values, lengths, cu, table, window, sinks, scale)
    mine = ~np.isnan(lse)
    score = (d + 4) * 2.0 ** -24 * np.where(mine, reach, 0.0)
    p_err = HALF_STEP + v_rel + 2 * score + 1e-5
    o = got_out[mine]
    assert np.isfinite(o).all(), "not finite"
    check_bf16(o, out[mine], (p_err[..., None] * np.where(np.isnan(spread), 0.0, spread))[mine], "out")
    if got_lse is not None:
        a, b = got_lse[mine], lse[mine]
        empty = np.isinf(b)
        assert (a[empty] == -np.inf).all()
        err = np.abs(a[~empty] - b[~empty])
        assert (err <= score[mine][~empty] + 4e-6 * (1 + np.abs(b[~empty]))).all(), err.max()
    return mine
