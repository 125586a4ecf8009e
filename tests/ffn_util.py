"""The residual feed-forward block's operators in 64 bits, by their formulas and on the CPU where sizes allow, for the tests."""
import numpy as np
import torch

from paper_2001_04206_amd import dn

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# unit roundoff: the largest relative error of one rounding
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
ACTS = {"linear": dn.DN_ACT_LINEAR, "sigmoid": dn.DN_ACT_SIGMOID, "tanh": dn.DN_ACT_TANH, "relu": dn.DN_ACT_RELU,
        "silu": dn.DN_ACT_SILU, "gelu": dn.DN_ACT_GELU}


def tolerance(dtype, terms, roundings=1):
    """Relative 2-norm error that `roundings` roundings to dtype of independent elements may leave, with the fp32 sums of `terms`
    products beneath them (their rounding errors add like a random walk, 2^-24 sqrt(terms), over a few more in the epilogue)
    and the 16-bit activations' 3e-7."""
    sums = 2.0 ** -24 * (terms ** 0.5 + 16)
    return sums if dtype == torch.float32 else roundings * UNIT[dtype] + sums + 3e-7


def close(got, want, tol, what):
    """2-norm within tol, and no element off by more than eight times that of itself or of the root mean square.  Few elements may
    be what is left of larger parts (everything the tests make is of size 1 to 4): they are held against those."""
    got, want = got.double().cpu(), want.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.isfinite(got).all(), what + ": not finite"
    off = (got - want).abs()
    norm = want.norm().item()
    if want.numel() < 64:
        norm = max(norm, 4 * want.numel() ** 0.5)
    rms = norm / want.numel() ** 0.5
    assert off.norm().item() <= tol * norm + 1e-30, "%s: %.3g of %.3g" % (what, off.norm().item() / max(norm, 1e-30), tol)
    worst = (off / want.abs().clamp(min=max(rms, 1e-30))).max().item()
    assert worst <= 8 * tol + 1e-30, "%s: an element is %.3g off, %.3g allowed" % (what, worst, 8 * tol)


def f64(z, act):
    z = z.double()
    return {"linear": lambda: z, "sigmoid": lambda: torch.sigmoid(z), "tanh": lambda: torch.tanh(z),
            "relu": lambda: z.clamp(min=0), "silu": lambda: z * torch.sigmoid(z),
            "gelu": lambda: z * 0.5 * torch.erfc(-z / 2 ** 0.5)}[act]()


def df64(z, act):
    z = z.double().detach().clone().requires_grad_()
    return torch.autograd.grad(f64(z, act).sum(), z)[0] if act != "relu" else (z > 0).double().detach()


def numbers(rows, cols, seed, offset):
    """Dropout's 16-bit numbers, [rows][cols], from the generator's definition in Python integers."""
    out = np.empty((rows, -(-cols // 8) * 8), np.int64)
    low = 2 ** 32 - 1
    for i in range(rows):
        for q in range(out.shape[1] // 8):
            c, k = [q, i, offset & low, offset >> 32], [seed & low, seed >> 32]
            for _ in range(10):
                p, r = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
                c = [r >> 32 ^ c[1] ^ k[0], r & low, p >> 32 ^ c[3] ^ k[1], p & low]
                k = [k[0] + 0x9E3779B9 & low, k[1] + 0xBB67AE85 & low]
            out[i, 8 * q:8 * q + 8] = [v for w in c for v in (w & 0xFFFF, w >> 16)]
    return out[:, :cols]


def mask64(rows, cols, drop, seed, offset):
    """What dropout multiplies by, [rows][cols]: the kernel's own answer for ones in fp32 (it is held against numbers() by a test
    of its own), which are exact."""
    if drop == 0:
        return torch.ones(rows, cols, dtype=torch.float64)
    x = torch.ones(rows, cols, device=DEV)
    dn.dn_dropout(x, x, drop, seed, offset)
    t = int(drop * 65536 + 0.5)
    return (x != 0).double().cpu() * (65536 / (65536 - t))


class Make:
    """Seeded normal tensors on the device; rows may lie `pad` elements further apart than they need to."""

    def __init__(self, dtype, seed):
        self.g, self.dtype = torch.Generator().manual_seed(seed), dtype

    def __call__(self, *shape, std=1.0, mean=0.0, pad=0):
        wide = shape[:-1] + (shape[-1] + pad,)
        t = (torch.randn(wide, generator=self.g) * std + mean).to(self.dtype).to(DEV)
        return t[..., :shape[-1]]

    def out(self, *shape, dtype=None):
        return torch.full(shape, float("nan"), dtype=dtype or self.dtype, device=DEV)
