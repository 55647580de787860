"""What surrounds a layer's products, from the definitions in 64 bits (on the CPU where nothing else is said), with how far a kernel that holds its sums in FP32 and
rounds once to BF16 may be from it.

A rounding to BF16 is off by at most 2^-8 of the value (2^-134 among the subnormals).  A sum of K terms in FP32, in any order,
is off by at most K 2^-23 of the sum of their magnitudes (2^-23: an addition that cuts instead of rounding)."""
import torch

ROUND, STEP, TINY = 2.0 ** -8, 2.0 ** -23, 2.0 ** -133


def norm(x, residual, weight, eps):
    """(y, tolerance, sum, tolerance)"""
    h = x.double().cpu()
    h = h if residual is None else h + residual.double().cpu()
    w = torch.ones(h.shape[1], dtype=torch.float64) if weight is None else weight.double().cpu()
    y = h / torch.sqrt(h.square().mean(1, keepdim=True) + eps) * w
    # the mean: K / T terms one after the other and log2 T more (at most 128 together), the square root halves its error; the
    # elements' sums, the inverse root and two products: eight steps
    return y, y.abs() * (ROUND + 72 * STEP) + TINY, h, h.abs() * (ROUND + STEP) + TINY


def e4m3_values(code, scale, device="cpu"):
    code = code.to(device).long()
    man, exp = code & 7, (code >> 3) & 15
    v = torch.where(exp == 0, man.double() * 2.0 ** -9, (8 + man).double() * torch.pow(2.0, (exp - 10).double()))
    v = torch.where((code & 127) == 127, torch.nan, torch.where(code >= 128, -v, v))
    return _scaled(v, scale.to(device))


def e2m1_values(q, scale, device="cpu"):
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device=device)
    q = q.to(device).long()
    return _scaled(torch.stack([grid[q & 15], grid[q >> 4]], dim=-1).flatten(-2), scale.to(device))


def _scaled(v, scale):
    s = torch.pow(2.0, scale.double() - 127)
    s[scale == 255] = torch.nan
    return v * s.repeat_interleave(32, dim=-1)


def _sums(x, w):
    """x w^T and the sums of magnitudes."""
    return x @ w.T, x.abs() @ w.abs().T


def product(x8, xs, q, s, bias=None, gate=False, residual=None, device="cpu"):
    """(y, tolerance).  Before the scaled matrix instruction adds the products of eight neighbours, it cuts each to a multiple of 2^-13 of
    the power of two of the largest (found by giving it 1024, -1024 and a third number: 2^-3 comes back, 2^-4 does not; 1.875 x 2^-2 comes back
    as 1.5 x 2^-2): seven of them are off by 2^-13 of the largest product at most, which is neither over the eight's sum of
    magnitudes nor over the product of their largest elements."""
    x, w = e4m3_values(x8, xs, device), e2m1_values(q, s, device)
    z, size = _sums(x, w)
    most = torch.minimum(size, x.abs().unflatten(1, (-1, 8)).amax(2) @ w.abs().unflatten(1, (-1, 8)).amax(2).T)
    off = (x.shape[1] + 1) * STEP * size + 7 * 2.0 ** -13 * most
    if bias is not None:
        z = z + bias.double().to(device)
        off = off + STEP * z.abs()
    if gate:
        g, u, og, ou = z[:, 0::2], z[:, 1::2], off[:, 0::2], off[:, 1::2]
        silu = g * torch.sigmoid(g)
        # silu's slope is below 1.1; e^-g through a power of two: its argument's rounding is off by 127 2^-24 at most
        z, off = silu * u, 1.1 * og * u.abs() + silu.abs() * ou + 1.1 * og * ou + (silu * u).abs() * 2.0 ** -16
    if residual is not None:
        z = z + residual.double().to(device)
        off = off + STEP * z.abs()
    return z, off + z.abs() * ROUND + TINY


def adapters(x, a, b, ids, base=None, scales=None):
    """(y, tolerance)"""
    x, a, b, ids = x.double().cpu(), a.double().cpu(), b.double().cpu(), ids.cpu()
    m, n, rank, k = x.shape[0], b.shape[1], a.shape[1], x.shape[1]
    y = torch.zeros((m, n), dtype=torch.float64) if base is None else base.double().cpu()
    off = torch.zeros((m, n), dtype=torch.float64)
    for i in range(a.shape[0]):
        rows = torch.nonzero(ids == i).flatten()
        if not rows.numel():
            continue
        f = 1.0 if scales is None else float(scales[i])
        t, size = _sums(x[rows], a[i])
        t, t_off = f * t, abs(f) * ((k + 1) * STEP * size + t.abs() * (2.0 ** -16 + STEP))
        d, d_size = _sums(t, b[i])
        y[rows] += d
        off[rows] = t_off @ b[i].abs().T + (2 * rank + 2) * STEP * d_size
    mine = (ids >= 0) & (ids < a.shape[0])
    return y, torch.where(mine[:, None], off * (1 + STEP) + y.abs() * (ROUND + STEP) + TINY, 0.0)


def near(got, want, tolerance, what=""):
    got = got.double().to(want.device)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "%s: NaN in other places" % what
    bad = torch.nonzero(~((got - want).abs() <= tolerance) & ~torch.isnan(want) & (got != want))
    assert not len(bad), "%s: %d of %d off, first at %r: %r for %r, tolerance %r" % (
        what, len(bad), got.numel(), tuple(bad[0].tolist()), float(got[tuple(bad[0])]), float(want[tuple(bad[0])]), float(tolerance[tuple(bad[0])]))
