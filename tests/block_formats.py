"""Blocks of 32 neighbours with a power of two as scale, from their definition in 64
bits: a table of every magnitude of the format, the smallest scale with which nothing
rounds past its largest, the nearest entry (ties to the even code)."""
import torch

BLOCK = 32
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
MOST = {torch.float32: torch.finfo(torch.float32).max, torch.float16: 65504.0, torch.bfloat16: float(torch.finfo(torch.bfloat16).max)}


def magnitudes(kind):
    """Every magnitude by code."""
    if kind == "i8":
        return [float(k) for k in range(128)]
    bits, bias, count = {"e4m3": (3, 7, 127), "e2m1": (1, 1, 8)}[kind]
    return [(c % 2 ** bits) * 2.0 ** (1 - bias - bits) if c < 2 ** bits else
            (1 + (c % 2 ** bits) / 2 ** bits) * 2.0 ** ((c >> bits) - bias) for c in range(count)]


def power(e):
    """2^e in 64 bits, exactly."""
    return torch.tensor([2.0 ** k for k in range(-300, 301)], dtype=torch.float64, device=e.device)[e.long() + 300]


def quantise(x, kind):
    """(values in 64 bits, scales' bytes) of x's rows; values are NaN where the block holds an infinity or NaN."""
    grid = torch.tensor(magnitudes(kind), dtype=torch.float64, device=x.device)
    n, d = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -d % BLOCK)).view(n, -(-d // BLOCK), BLOCK)
    fine = v.isfinite().all(2, keepdim=True)
    v = torch.where(fine, v, 0.0)

    def nearest(u):
        u = u.contiguous()
        mid = (grid[1:] + grid[:-1]) / 2
        low, high = torch.searchsorted(mid, u), torch.searchsorted(mid, u, right=True)
        return grid[torch.where((low != high) & (low % 2 == 1), high, low)]

    amax = v.abs().amax(2, keepdim=True)
    # the next magnitude that a format without a largest would have, and where it begins
    after = grid[-1] + (grid[-1] - grid[-2])
    begins = (grid[-1] + after) / 2
    tie_up = kind != "e4m3"  # 127.5 -> 128 and 7 -> 8 are even, 464 -> 448
    e = torch.full_like(amax, -127, dtype=torch.int64)
    for k in range(-126, 128):
        u = amax / 2.0 ** (k - 1)
        e = torch.where((u >= begins) if tie_up else (u > begins), k, e)
    s = power(e)
    value = torch.sign(v) * nearest(v.abs() / s) * s
    value = torch.where(fine, value, float("nan")).reshape(n, v.shape[1] * BLOCK)[:, :d]
    return value, torch.where(fine[:, :, 0], e[:, :, 0] + 127, 255).to(torch.uint8)


def decode(codes, scales, kind, d):
    """The values that codes and scales stand for, in 64 bits."""
    if kind == "e2m1":
        grid = torch.tensor(magnitudes(kind), dtype=torch.float64, device=codes.device)
        half = torch.stack((codes & 15, codes >> 4), 2).flatten(1).long()
        flat = grid[half & 7] * (1 - 2 * (half >> 3)).double()
    else:
        flat = codes.float().double()
    scales = scales[:, :-(-d // BLOCK)]
    s = torch.where(scales == 255, float("nan"), power(scales.int() - 127))
    return (flat.view(len(codes), s.shape[1], BLOCK) * s[:, :, None]).flatten(1)[:, :d]


def rounded(value, dtype):
    """Values in a type, those past its largest as that."""
    return torch.where(value.isnan(), value, value.clamp(-MOST[dtype], MOST[dtype])).to(dtype)


def samples(n, d, dtype, device, seed, special=True):
    """Rows of sizes far apart, and rows at the formats' edges."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    x = torch.randn(n, d, generator=g, device=device, dtype=torch.float64)
    x = x * torch.exp(2.0 * torch.randn(n, 1, generator=g, device=device, dtype=torch.float64))
    if special and n >= 16:
        most = MOST[dtype]
        x[0] = 0
        x[1] *= 1e-30
        x[2] = x[2] * 1e-42
        x[3] = torch.randint(-31, 32, (d,), generator=g, device=device).double() * 0.25  # ties
        for row, edge in ((4, 127.5), (5, 127.49), (6, 464.0), (7, 466.0), (8, 7.0), (9, 6.99), (10, most)):
            x[row] = x[row].clamp(-1, 1) * 0.9 * edge
            x[row, ::7] = edge
        x[11, 0] = float("inf")
        x[12, d - 1] = float("nan")
        x[13, d // 2] = -float("inf")
    return x.to(dtype)


def strided(rows, cols, dtype, dev, pad=0, shift=0, fill=7):
    """A (rows, cols) tensor whose rows are cols + pad apart, `shift` elements into its memory."""
    base = torch.full((shift + max(rows, 1) * (cols + pad),), fill, dtype=dtype, device=dev) if dtype != torch.float8_e4m3fn else \
        torch.full((shift + max(rows, 1) * (cols + pad),), fill, dtype=torch.uint8, device=dev).view(dtype)
    return base[shift:][:rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
