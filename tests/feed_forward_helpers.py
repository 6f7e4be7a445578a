"""Plain 64-bit forms of a linear with an epilogue, a router and a mixture of experts, with bounds on what 32-bit sums may add."""
import math

import torch

# A rounding to float16 is off by half a step: 2^-11 of the value, or 2^-25 where it is subnormal.
HALF_STEP, SUBNORMAL = 2.0 ** -11, 2.0 ** -25
# A sum of K products in binary32, in any order and with truncated steps, is off by at most K 2^-23 sum |x w|.
STEP = 2.0 ** -23


def generator(seed, device="cuda:0"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g


def normal(g, *shape, sigma=1.0):
    return torch.empty(shape, dtype=torch.float16, device=g.device).normal_(0.0, sigma, generator=g)


def e4m3(x):
    """Values of E4M3 codes (uint8) in 64 bits."""
    return x.view(torch.float8_e4m3fn).double()


def upper_values(w):
    """What FP8 mode multiplies: E4M3 of 256 w, over 256."""
    return (w.float() * 256.0).to(torch.float8_e4m3fn).double() / 256.0


def quantized(x):
    """(codes as values, scales): per row, as the library defines them."""
    amax = x.abs().amax(1).float()
    # (a division by a tensor: by a number, torch multiplies by its reciprocal)
    scale = torch.where(amax == 0, torch.ones_like(amax), amax / torch.full_like(amax, 448.0))
    return (x.float() / scale[:, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), scale


def activated(z, act):
    if act == 1:
        return z.clamp(min=0.0)
    if act == 2:
        return z * torch.sigmoid(z)
    if act == 3:
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


# Slopes of the activations are at most 1.13; exponential, reciprocal and their arguments are off by less than 2^-17 of the result (|u| < 2^7).
SLOPE, ACT_ERROR = 1.13, 2.0 ** -17


def epilogue_ref(z, off, bias, act, gated, residual):
    """(y, tolerance) from the sums z, which are off by `off`; gated: rows in turn along the columns of z."""
    if bias is not None:
        z = z + bias.double()
        off = off + z.abs() * STEP
    if gated:
        a, up = activated(z[:, 0::2], act), z[:, 1::2]
        y = a * up
        off = (off[:, 0::2] * SLOPE + a.abs() * ACT_ERROR) * (up.abs() + off[:, 1::2]) + a.abs() * off[:, 1::2] + y.abs() * STEP
    else:
        y = activated(z, act)
        off = off * SLOPE + (y.abs() * ACT_ERROR if act else 0.0)
    if residual is not None:
        y = y + residual.double()
        off = off + y.abs() * STEP
    return y, off + (y.abs() + off) * HALF_STEP + SUBNORMAL


def linear_ref(x, w, fp8, bias=None, act=0, gated=False, residual=None):
    """The reference of linear_fused; w in the order of the layer's rows."""
    if fp8:
        codes, scale = quantized(x)
        wide, w = codes.double() * scale.double()[:, None], upper_values(w)
    else:
        wide, w = x.double(), w.double()
    z, size = wide @ w.t().contiguous(), wide.abs() @ w.abs().t().contiguous()
    return epilogue_ref(z, (x.shape[1] + 4) * STEP * size, bias, act, gated, residual)


def assert_within(got, ref, tol, what=""):
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bad.any(), "%s: %d of %d outside, at %s: %s for %s" % (
        what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), got[bad][0].item(), ref[bad][0].item())


def moe_ref(x, gate_up, down, ids, weights, fp8, act, residual=None):
    """(y, tolerance) of a mixture of experts; gate rows first.  The activated products are kept to 2^-22."""
    experts, hidden, ffn = down.shape
    m = x.shape[0]
    y = torch.zeros((m, hidden), dtype=torch.float64, device=x.device) if residual is None else residual.double().clone()
    off, size = torch.zeros_like(y), y.abs().clone()
    wide, value = x.double(), (upper_values if fp8 else (lambda w: w.double()))
    for t in range(m):
        for j in range(ids.shape[1]):
            e = int(ids[t, j])
            if not 0 <= e < experts:
                continue
            w1, w2, share = value(gate_up[e]), value(down[e]), float(weights[t, j])
            z, zs = w1 @ wide[t], w1.abs() @ wide[t].abs()
            dz = (hidden + 4) * STEP * zs
            a, up = activated(z[:ffn], act), z[ffn:]
            h = a * up
            dh = (dz[:ffn] * SLOPE + a.abs() * ACT_ERROR) * (up.abs() + dz[ffn:]) + a.abs() * dz[ffn:] + h.abs() * 2.0 ** -21 + 2.0 ** -25
            y[t] += share * (w2 @ h)
            size[t] += abs(share) * (w2.abs() @ h.abs())
            off[t] += abs(share) * (w2.abs() @ dh)
    off = off + (2 * ffn + 4 * ids.shape[1] + 8) * STEP * size
    return y, off + (y.abs() + off) * HALF_STEP + SUBNORMAL


def route_ref(x, router, top_k, sigmoid, renormalize, bias, factor):
    """(ids, weights) on the host in 64 bits; the lowest index first of equal choices."""
    logits = x.double().cpu() @ router.double().cpu().t()
    score = torch.sigmoid(logits) if sigmoid else torch.softmax(logits, 1)
    choice = logits if bias is None else score + bias.double().cpu()
    ids = torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :top_k]
    weights = score.gather(1, ids)
    if renormalize:
        weights = weights / weights.sum(1, keepdim=True)
    return ids.to(torch.int32), weights * factor
