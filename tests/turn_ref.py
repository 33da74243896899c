"""Plain 64-bit implementation of the norms and rotations (torch on the CPU), and the bounds that outputs are held to."""
import torch


def table(positions, dim, base=10000.0):
    """The documented table: cosines and behind them sines of dim / 2 pairs, float32."""
    angle = torch.arange(positions, dtype=torch.float64).unsqueeze(1) * base ** (-torch.arange(dim // 2, dtype=torch.float64) * 2 / dim)
    return torch.cat((angle.cos(), angle.sin()), 1).float().contiguous()


def turned(x, weight, eps, angles, positions, neighbours):
    """Rows x [n][heads][D] normalised and turned -> rows and sizes in 64 bits: |a cos| + |b sin| of each element, which errors are relative to."""
    x = x.double()
    if weight is not None:
        root = torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        x = torch.where(root > 0, x / torch.where(root > 0, root, 1), 0.0) * weight.double()
    y, size = x.clone(), x.abs()
    if angles is not None:
        dim = angles.shape[1]
        at = torch.arange(dim // 2)
        first, second = (2 * at, 2 * at + 1) if neighbours else (at, at + dim // 2)
        known = (positions >= 0) & (positions < angles.shape[0])
        rows = angles[torch.where(known, positions, 0).long()].double().unsqueeze(1)
        c, s, a, b = rows[..., :dim // 2], rows[..., dim // 2:], x[..., first], x[..., second]
        y[..., first], y[..., second] = a * c - b * s, b * c + a * s
        size[..., first], size[..., second] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
        y[~known] = torch.nan
    return y, size


# Arithmetic in float: the sum of squares is off by at most 16 + 4 roundings (16 elements a lane, sums over lanes) and those of the mean and eps, its root by half of
# that; root, quotient, two products, then a product and a sum of two: less than 20 roundings of 2^-24, doubled for what 64 bits count as first order only.
ARITHMETIC = 40 * 2.0 ** -24
# unit roundoffs, and half the distance of the smallest numbers
U = {torch.float32: (2.0 ** -24, 2.0 ** -149), torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 2.0 ** -133)}


def check_rows(got, want, size):
    u, least = U[got.dtype]
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    off = ((got - want).abs() - (u * want.abs() + (1 + u) * ARITHMETIC * size + least)).nan_to_num(-1.0)
    assert off.numel() == 0 or float(off.max()) <= 0, f"{float(off.max())} past the bound"
