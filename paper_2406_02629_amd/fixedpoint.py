"""Plaintext side of the harness: fixed-point encode / decode between float64
tensors and field elements (Sec. II-B: F_p stands for the signed range
[-(p-1)/2, (p-1)/2]; values are scaled by 2^f and rounded to nearest-even).
These run on the data owner's side, outside the share arithmetic.
"""
import torch

P61 = (1 << 61) - 1


def encode(x: torch.Tensor, f: int, p: int = P61) -> torch.Tensor:
    """float64 -> field elements as int64: round-half-even(x * 2^f) mod p."""
    v = torch.round(x.to(torch.float64) * float(1 << f))
    if bool((v.abs() >= float(1 << 40)).any()):
        raise ValueError("value exceeds 2^40 after scaling")
    v = v.to(torch.int64)
    return torch.where(v < 0, v + p, v)


def lift(u: torch.Tensor, p: int = P61) -> torch.Tensor:
    """field element -> signed integer: u if u <= (p-1)/2 else u - p."""
    return torch.where(u > (p - 1) // 2, u - p, u)


def from_signed(v: torch.Tensor, p: int = P61) -> torch.Tensor:
    return torch.where(v < 0, v + p, v)


def decode(u: torch.Tensor, s: int, p: int = P61) -> torch.Tensor:
    """field element -> float64 lift(u) / 2^s."""
    return lift(u, p).to(torch.float64) / float(1 << s)


def rotary_frequencies(rot: int, base: float = 10000.0, factor: float = 1.0, original: int = 0, low: float = 1.0,
                       high: float = 4.0) -> torch.Tensor:
    """Angles per position of the rot / 2 pairs of a head, base^(-2j/rot), float64.  factor > 1 stretches them for contexts that
    are `factor` times longer: all of them (original = 0), or, with `original` the context length of the training, those
    that turn at most `low` times in it, none that turn `high` times or more, and a mixture between."""
    if rot < 2 or rot % 2 or base <= 0 or factor < 1:
        raise ValueError("rot must be even, base positive, factor at least 1")
    freq = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if original == 0:
        return freq / factor
    if not 0 < low < high:
        raise ValueError("0 < low < high")
    keep = ((original * freq / (2 * torch.pi) - low) / (high - low)).clamp(0.0, 1.0)
    return keep * freq + (1 - keep) * freq / factor


def rotary_table(positions: int, frequencies: torch.Tensor, f: int, magnitude: float = 1.0, device=None) -> torch.Tensor:
    """int32 [positions][rot / 2][2]: round(2^f magnitude cos), round(2^f magnitude sin) of the angles at positions 0, 1, ..."""
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * frequencies.to(torch.float64)
    t = torch.stack([angle.cos(), angle.sin()], -1) * (magnitude * (1 << f))
    if bool((t.abs() >= 2.0 ** 31).any()):
        raise ValueError("the table does not fit 32 bits")
    return torch.round(t).to(torch.int32).to(device).contiguous()


def sampling_parameters(temperature, top_k=0, top_p=1.0, min_p=0.0, rows: int = 1, device=None) -> torch.Tensor:
    """int32 [rows][4] for SSNet.sample, each argument a number or one for every row: temperature 0.0113 to 1477 (0: the most likely token), top_k
    (0: all), top_p and min_p between 0 and 1"""
    def column(v, name, low, high):
        t = torch.as_tensor(v, dtype=torch.float64)
        if t.dim() > 1 or (t.dim() == 1 and t.shape[0] != rows):
            raise ValueError(f"{name} must be a number or one for each of {rows} rows")
        if not bool(((t >= low) & (t <= high)).all()):
            raise ValueError(f"{name} must lie between {low} and {high}")
        return t.expand(rows)

    t = column(temperature, "temperature", 0, 1477)
    if bool(((t > 0) & (t < 0.0113)).any()):
        raise ValueError("temperature must be 0 or at least 0.0113")
    scale = torch.where(t > 0, (2.0 ** 24 / 0.6931471805599453 / t.clamp(min=0.0113)).round(), 0)
    k = column(top_k, "top_k", 0, 2 ** 31 - 1)
    if bool((k != k.round()).any()):
        raise ValueError("top_k must be a whole number")
    p, m = (2.0 ** 30 * column(v, name, 0, 1) for v, name in ((top_p, "top_p"), (min_p, "min_p")))
    return torch.stack([scale, k, p.round(), m.round()], 1).to(torch.int32).to(device).contiguous()
