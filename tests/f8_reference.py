"""The 8-bit form and the products on it from their definitions, in 64 bits."""
import torch

BLOCK = 128


def exponents(x, tall=1):
    """The scales' bytes [blocks of rows, blocks of columns] of a 64-bit tensor."""
    r, c = x.shape
    full = torch.zeros(-(-r // tall) * tall, -(-c // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    full[:r, :c] = x
    amax = full.view(-1, tall, full.shape[1] // BLOCK, BLOCK).abs().amax((1, 3))
    b = torch.full_like(amax, 1.0)
    for k in range(2, 255):  # the smallest power of two that brings the largest to 448 at most
        b = torch.where(amax > 448.0 * 2.0 ** (k - 1 - 127), float(k), b)
    b = torch.where(amax == 0, 127.0, b)
    return torch.where(torch.isfinite(amax), b, 255.0).to(torch.int64)


def spread(b, shape, tall=1):
    return b.repeat_interleave(tall, 0)[:shape[0]].repeat_interleave(BLOCK, 1)[:, :shape[1]]


def codes(y):
    """The E4M3 values next to y (|y| <= 448), ties to even."""
    unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / unit) * unit


def form(x, tall=1):
    """(codes' values, scales' bytes) of the 8-bit form of x."""
    x = x.double()
    b = exponents(x, tall)
    scale = torch.where(spread(b, x.shape, tall) == 255, torch.nan, torch.exp2(spread(b, x.shape, tall).double() - 127))
    return codes(x / scale), b


def value(c, b, tall=1):
    """What codes and scales' bytes stand for."""
    s = spread(b.long(), c.shape, tall)
    return c.double() * torch.where(s == 255, torch.nan, torch.exp2(s.double() - 127))


def meant(f, transposed=False):
    """The values of an F8Rows, or of one orientation of an F8Weight."""
    if transposed:
        return value(f.codes_t.double(), f.scales_t.view(torch.uint8), BLOCK)
    return value(f.codes.double(), f.scales.view(torch.uint8), BLOCK if hasattr(f, "codes_t") else 1)


def gelu(u, kind):
    return torch.nn.functional.gelu(u, approximate="tanh" if kind == "tanh" else "none")


def gelu_grad(u, kind):
    u = u.clone().requires_grad_()
    return torch.autograd.grad(gelu(u, kind).sum(), u)[0]
