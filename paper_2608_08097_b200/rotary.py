"""Frequencies of rotary positions, with the usual ways to stretch them over contexts longer than the trained one.

A table is made once per model and handed to `binding.rotate_qkv`; the angles themselves are computed on the GPU, in 64 bits.
"""
import math

import torch


def _yarn(rot_dim, base, factor, trained, beta_fast=32.0, beta_slow=1.0, attention_factor=None):
    """Frequencies that turn less than beta_slow times over the trained positions are divided by `factor`, those that turn more than
    beta_fast times stay, with a linear ramp over the dims between; cos and sin grow by 0.1 ln(factor) + 1."""
    if not beta_fast > beta_slow > 0:
        raise ValueError("scaling 'yarn': beta_fast above beta_slow above zero")

    def dim_of(turns):
        return rot_dim * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))

    low, high = max(math.floor(dim_of(beta_fast)), 0), min(math.ceil(dim_of(beta_slow)), rot_dim - 1)
    f = _plain(rot_dim, base)
    ramp = ((torch.arange(rot_dim // 2, dtype=torch.float64) - low) / max(high - low, 0.001)).clamp(0, 1)
    if attention_factor is None:
        attention_factor = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    return f / factor * ramp + f * (1 - ramp), attention_factor


def _bands(rot_dim, base, factor, trained, low_freq_factor=1.0, high_freq_factor=4.0):
    """Wavelengths longer than trained / low_freq_factor are stretched by `factor`, those shorter than trained / high_freq_factor
    stay, and between them the two are blended."""
    if not high_freq_factor > low_freq_factor > 0:
        raise ValueError("scaling 'bands': high_freq_factor above low_freq_factor above zero")
    f = _plain(rot_dim, base)
    turns = trained * f / (2 * math.pi)                          # over the trained positions
    blend = ((turns - low_freq_factor) / (high_freq_factor - low_freq_factor)).clamp(0, 1)
    return (1 - blend) * f / factor + blend * f, 1.0


def _plain(rot_dim, base):
    return base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)


class RotaryTable:
    """Frequencies (radians per position, fp64, on `device`) and the factor on cos and sin.

    rot_dim      dims of a head that are rotated (even, at most 128); the others are copied
    interleaved  pairs (2i, 2i + 1) instead of (i, i + rot_dim / 2)
    scaling      None, or a dict with "kind" and its parameters:
        "linear"  factor                     positions divided by `factor`
        "ntk"     factor                     a larger base, so that the slowest frequency is divided by `factor`, the fastest stays
        "yarn"    factor, trained, beta_fast=32, beta_slow=1, attention_factor=None
        "bands"   factor, trained, low_freq_factor=1, high_freq_factor=4
        "given"   factors [rot_dim / 2], attention_factor=1    every frequency divided by its own factor
    """

    def __init__(self, rot_dim=128, base=10000.0, interleaved=False, scaling=None, device="cuda"):
        if rot_dim % 2 or not 2 <= rot_dim <= 128:
            raise ValueError("rot_dim %d: an even number from 2 to 128" % rot_dim)
        if not base > 1:
            raise ValueError("base %g: above 1" % base)
        p = dict(scaling or {"kind": "none"})
        kind = p.pop("kind", None)
        if kind in ("linear", "ntk", "yarn", "bands") and not p.get("factor", 0) > 0:
            raise ValueError("scaling %r needs a factor above zero" % kind)
        if kind in ("yarn", "bands") and not p.get("trained", 0) > 0:
            raise ValueError("scaling %r needs the number of trained positions" % kind)
        try:
            freqs, factor = self._frequencies(kind, rot_dim, float(base), p)
        except TypeError as e:
            raise ValueError("scaling %r: %s" % (kind, e)) from e
        self.rot_dim, self.interleaved, self.factor = int(rot_dim), int(bool(interleaved)), float(factor)
        self.freqs = freqs.to(device)

    @staticmethod
    def _frequencies(kind, rot_dim, base, p):
        if kind == "none" and not p:
            return _plain(rot_dim, base), 1.0
        if kind == "linear" and set(p) == {"factor"}:
            return _plain(rot_dim, base) / p["factor"], 1.0
        if kind == "ntk" and set(p) == {"factor"}:
            return _plain(rot_dim, base * p["factor"] ** (rot_dim / max(rot_dim - 2, 1))), 1.0
        if kind == "yarn":
            return _yarn(rot_dim, base, **p)
        if kind == "bands":
            return _bands(rot_dim, base, **p)
        if kind == "given" and "factors" in p and set(p) <= {"factors", "attention_factor"}:
            f = torch.as_tensor(p["factors"], dtype=torch.float64, device="cpu").flatten()
            if f.numel() != rot_dim // 2 or not bool((f > 0).all()):
                raise ValueError("scaling 'given': %d factors above zero are needed" % (rot_dim // 2))
            return _plain(rot_dim, base) / f, p.get("attention_factor", 1.0)
        raise ValueError("scaling %r with %s is not known" % (kind, sorted(p)))
