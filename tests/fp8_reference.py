"""Plain 64-bit definitions of the operators for 8-bit layers and clipping, for the tests."""
import torch

DEV = "cuda:0"
DT = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}
STEP = {"e4m3": 2.0 ** -4, "e5m2": 2.0 ** -3}        # half a step, relative to the value
LEAST = {"e4m3": 2.0 ** -10, "e5m2": 2.0 ** -17}     # half of the smallest step


def expand(scale, block_rows, rows, cols):
    return scale.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def block_amax(x, block_rows):
    """The largest finite magnitude of each block of x (float64)."""
    rows, cols = x.shape
    rb, cb = -(-rows // block_rows), -(-cols // 128)
    p = torch.zeros(rb * block_rows, cb * 128, dtype=torch.float64)
    p[:rows, :cols] = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    return p.view(rb, block_rows, cb, 128).amax(dim=(1, 3))


def quantise(x, block_rows, fmt):
    """(data in 8 bits, scale bytes) of x, any float type, on the CPU."""
    x = x.detach().double().cpu()
    amax = block_amax(x, block_rows)
    e = torch.full_like(amax, -127.0)
    for k in range(-126, 128):           # the least e with amax <= TOP 2^e, at least -127
        e = torch.where(amax > TOP[fmt] * 2.0 ** (k - 1), torch.full_like(e, float(k)), e)
    e = torch.where(amax == 0, torch.zeros_like(e), e)
    s = expand(torch.pow(2.0, e), block_rows, *x.shape)
    return (x / s).float().to(DT[fmt]), (e + 127).to(torch.uint8)


def wide(f):
    """What an Fp8 stands for, float64 on the CPU."""
    return f.data.cpu().to(torch.float32).double() * expand(f.scale.cpu().to(torch.float32).double(), f.block_rows, *f.shape)


def norm_forward(total, gain, eps, norm):
    total, gain = total.double(), gain.double()
    c = total - total.mean(1, keepdim=True) if norm == "layer" else total
    rstd = 1.0 / torch.sqrt((c * c).mean(1) + eps)
    return c * rstd[:, None] * gain, rstd


def norm_backward(dy, total, rstd, gain, norm):
    """(ds without ds_in, dgain)"""
    dy, total, rstd, gain = dy.double(), total.double(), rstd.double()[:, None], gain.double()
    xh = (total - total.mean(1, keepdim=True) if norm == "layer" else total) * rstd
    h = dy * gain
    ds = rstd * (h - (h.mean(1, keepdim=True) if norm == "layer" else 0.0) - xh * (h * xh).mean(1, keepdim=True))
    return ds, (dy * xh).sum(0)
