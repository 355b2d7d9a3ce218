"""Rotary positions of one model: the table of frequencies and the call."""

from __future__ import annotations

import torch

from . import _lib


class RotaryPositions:
    """Rotates queries and keys by their positions.

    rotary_dim: how many channels of every head turn (the first ones).
    layout: "half" pairs channel i with i + rotary_dim / 2, "interleaved" 2 i
    with 2 i + 1.
    scaling: "none"; "linear" and "ntk" with a factor; "bands" and "yarn" with a
    factor, the original context and turns = (turns_low, turns_high), by default
    (1, 4) and (1, 32).
    magnitude: the factor of the rotated values, the scaling's own if None."""

    def __init__(self, rotary_dim: int = 128, base: float = 10000.0, layout: str = "half", scaling: str = "none",
                 factor: float = 1.0, original: float = 0.0, turns=None, magnitude=None, device="cuda"):
        if layout not in _lib.ROPE_LAYOUTS:
            raise ValueError("layout must be 'half' or 'interleaved'")
        if turns is None:
            turns = (1.0, 32.0) if scaling == "yarn" else (1.0, 4.0)
        freq, own = _lib.dq_rope_frequencies(rotary_dim, base, scaling, factor, original, turns)
        self.rotary_dim, self.layout = rotary_dim, layout
        self.magnitude = own if magnitude is None else float(magnitude)
        self.freq = torch.from_numpy(freq).to(device)      # fp64 [rotary_dim / 2]

    def apply(self, q=None, k=None, positions=None, starts=None, t0: int = 0, transposed: bool = False, q_out=None,
              k_out=None, stream=None):
        """q bf16 [B, T, Hq, d], k bf16 [B, T, Hkv, d] (either may be None) at
        int32 positions [B, T], or at t0 + t plus int32 starts [B] (the lengths
        of a cache).  Returns (q_out, k_out): new tensors unless given; the
        inputs themselves rotate in place.  transposed: the transposed map, the
        gradient of the inputs from that of the outputs."""
        return _lib.dq_rope(self.freq, q, k, positions, starts, t0, self.layout, transposed, self.magnitude, q_out,
                            k_out, stream)
