"""What the tests of the operators share."""
import torch


def rounds_from(out: torch.Tensor, want: torch.Tensor, slack: torch.Tensor) -> torch.Tensor:
    """Whether each value of `out` is what some number within `slack` of `want` (both in 64 bits) rounds to in out's
    type: rounding is monotone, so it lies between the roundings of the two ends.  No tolerance for the rounding itself."""
    lo, hi = ((want + s).float().to(out.dtype).double() for s in (-slack, slack))
    out = out.double()
    return (lo <= out) & (out <= hi)
