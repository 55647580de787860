"""The product of 8-bit rows on the GPU, its larger blocks (gemm_a8_mid.hip, gemm_a8_block.hip) above all, against the definition in 64 bits (layer_plain.py).  Which
block a call takes follows from its sizes and the device's units; the sizes here are for 256 of them."""
import pytest
import torch

import layer_plain as plain
from paper_2503_13565_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _bf16(shape, seed, scale=1.0, large=20.0):
    x = torch.randn(shape, generator=_gen(seed)) * scale
    x[..., 3] *= large
    return x.to(torch.bfloat16).to(DEV)


@pytest.mark.parametrize("m,n,k", [
    (33, 8193, 96), (35, 8195, 32), (193, 8194, 64), (33, 4097, 1376),              # blocks of 32 x 64
    (129, 8193, 160), (65, 12289, 416), (257, 4097, 96),                             # of 64 x 128
    (257, 8193, 96), (258, 8194, 32), (257, 8193, 1376)])                            # of 128 x 128
def test_product_of_a_last_block_of_a_row_and_a_column(m, n, k):
    """Blocks with a row or two, a weight row or two, and a K that is no multiple of an instruction's: less memory than a phase of whole steps."""
    x8, xs = binding.mxfp4_e4m3_direct_cast(_bf16((m, k), 1))
    q, s = binding.mxfp4_direct_cast(_bf16((n, k), 2, 0.05, 4.0))
    y = binding.mxfp4_w4a8_gemm(x8, xs, q, s)
    plain.near(y, *plain.product(x8, xs, q, s, device=DEV))


@pytest.mark.parametrize("m", [2, 9, 30, 300])
def test_product_of_a_closed_gate(m):
    """Gates from -86 to -88.5, whose silu is 2^-118 and less, beside numbers that bring it back; some at the other ends of FP32.  Codes of zero, so that
    the sums are the bias."""
    n, k = 9000 if m > 30 else 200, 64
    bias = torch.empty((n,), device=DEV)
    bias[0::2] = torch.tensor([-86, -86.5, -87, -87.5, -88, -88.5, 3e38, 1e-36], device=DEV).repeat(n // 16 + 1)[: n // 2]
    bias[1::2] = 1.0e38 * (1 + torch.arange(n // 2, device=DEV) % 5 * 0.5)
    bias[13::16] = 0.5
    bias = bias.to(torch.bfloat16)
    x8, xs = torch.zeros((m, k), dtype=torch.uint8, device=DEV), torch.full((m, k // 32), 127, dtype=torch.uint8, device=DEV)
    q, s = torch.zeros((n, k // 2), dtype=torch.uint8, device=DEV), torch.full((n, k // 32), 127, dtype=torch.uint8, device=DEV)
    y = binding.mxfp4_w4a8_gemm(x8, xs, q, s, bias=bias, act=binding.ACT_SWIGLU)
    g, u = bias.double()[0::2], bias.double()[1::2]
    want = (g * torch.sigmoid(g) * u).expand(m, -1)
    # e^-g through a power of two whose argument (128 at most) is rounded: 127 2^-24; the power, the reciprocal and the products: a step or two each
    plain.near(y, want, want.abs() * (2.0 ** -16 + plain.ROUND))


@pytest.mark.parametrize("m,gate", [(1, False), (1, True), (20, False)])
def test_product_of_more_weight_rows_than_a_launch_has(m, gate):
    """Grids of sixteen weight rows a workgroup end at 2^27.  Ones against any codes: sums of 32 multiples of 1/2, exact."""
    n, k = (1 << 27) + 54, 32
    gen = torch.Generator(device=DEV).manual_seed(m)
    q = torch.randint(0, 256, (n, k // 2), generator=gen, dtype=torch.uint8, device=DEV)
    s = torch.randint(126, 129, (n, 1), generator=gen, dtype=torch.uint8, device=DEV)
    x8, xs = torch.full((m, k), 0x38, dtype=torch.uint8, device=DEV), torch.arange(m, dtype=torch.int32, device=DEV)[:, None]
    c = n // 2 if gate else n
    bias = torch.randint(-4, 5, (n,), generator=gen, device=DEV).to(torch.bfloat16)
    residual = torch.randint(-4, 5, (m, c), generator=gen, dtype=torch.int8, device=DEV).to(torch.bfloat16)
    y = binding.mxfp4_w4a8_gemm(x8, (127 - xs % 3).to(torch.uint8), q, s, bias=bias, act=binding.ACT_SWIGLU if gate else binding.ACT_NONE, residual=residual)
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    two = grid.repeat(16) + grid.repeat_interleave(16)
    scale = torch.exp2(-(xs % 3).float())
    for at in range(0, n, 1 << 22):
        z = (two[q[at : at + (1 << 22)].int()].sum(1) * torch.exp2(s[at : at + (1 << 22), 0].float() - 127))[None] * scale + bias[at : at + (1 << 22)].float()
        off = torch.zeros_like(z)
        if gate:
            g, u = z.double()[:, 0::2], z.double()[:, 1::2]
            z = g * torch.sigmoid(g) * u
            # e^-g and the products around it: see the closed gates; below -88.72 e^-g is no FP32 number and the gate is 0, where
            # |g| / (1 + e^-g) falls as g does and is less than 88.8 2^-128 < 2^-121
            off = 2.0 ** -16 * z.abs() + (g < -88.72) * 2.0 ** -121 * u.abs()
        lo = at // 2 if gate else at
        z = z + residual[:, lo : lo + z.shape[1]]
        off = off + (plain.ROUND + plain.STEP * gate) * z.abs()
        bad = torch.nonzero(~((y[:, lo : lo + z.shape[1]].double() - z.double()).abs() <= off.double()))
        assert not len(bad), "%d off behind %d, first at %r: %r for %r" % (len(bad), lo, bad[0].tolist(), float(y[bad[0][0], lo + bad[0][1]]), float(z[tuple(bad[0])]))


BLOCKS = [(17, 66), (17, 8194), (35, 8197), (98, 8195), (227, 8194), (258, 7237), (449, 8201), (1025, 7170)]     # every block where K is some thousands


def _whole(shape, most, gen):
    """Whole numbers -most .. most (at most 4) and half of them zeros: as values, as E4M3 codes, as E2M1 codes."""
    v = torch.randint(-most, most + 1, shape, generator=gen, device=DEV)
    v = torch.where(torch.rand(shape, generator=gen, device=DEV) < 0.5, 0, v)
    eight = torch.tensor([0, 0x38, 0x40, 0x44, 0x48], dtype=torch.uint8, device=DEV)[v.abs()] | (v < 0).to(torch.uint8) << 7
    four = torch.tensor([0, 2, 4, 5, 6], dtype=torch.uint8, device=DEV)[v.abs()] | (v < 0).to(torch.uint8) << 3
    return v.double(), eight, four


@pytest.mark.parametrize("k", [160, 2080, 4128, 16416])
@pytest.mark.parametrize("m,n", BLOCKS)
def test_product_of_whole_numbers(m, n, k):
    """Whole numbers under scales of 1/2 to 2: products are multiples of 1/4, and eight neighbours, which share their scales, are nothing that the instruction
    cuts; sums of magnitudes stay below 2^23 of those, so FP32 holds every sum on the way, and every output is the exact sum rounded once."""
    gen = torch.Generator(device=DEV).manual_seed(m + n + k)
    (x, x8, _), (w, _, w4) = _whole((m, k), 4, gen), _whole((n, k), 4, gen)
    xs, ws = (torch.randint(126, 129, (rows, k // 32), generator=gen, device=DEV) for rows in (m, n))
    q = w4[:, 0::2] | w4[:, 1::2] << 4
    y = binding.mxfp4_w4a8_gemm(x8, xs.to(torch.uint8), q, ws.to(torch.uint8))
    x *= torch.exp2(xs.double() - 127).repeat_interleave(32, dim=1)
    w *= torch.exp2(ws.double() - 127).repeat_interleave(32, dim=1)
    want = x @ w.T
    assert 4 * 64 * k < 2 ** 23 and torch.equal(want, want.float().double())
    want = want.to(torch.float32).to(torch.bfloat16)
    bad = torch.nonzero(y != want)
    assert not len(bad), "%d off, first at %r: %r for %r" % (len(bad), bad[0].tolist(), float(y[tuple(bad[0])]), float(want[tuple(bad[0])]))


@pytest.mark.parametrize("k", [160, 4128])
@pytest.mark.parametrize("m,n", BLOCKS)
def test_product_of_every_scale_byte(m, n, k):
    """A row has a number in one place, weights are 1 and -1, and scale bytes are any: every output is the product of the two scales of that place's block,
    exact in BF16.  Rows that hold a NaN or the byte 0xFF, and weight rows with that byte, are NaN, and no others."""
    gen = torch.Generator(device=DEV).manual_seed(m + n + k)
    rows, nblk = torch.arange(m, device=DEV), k // 32
    at = (rows * 32 + rows % 32) % k
    x8 = torch.zeros((m, k), dtype=torch.uint8, device=DEV)
    x8[rows, at] = 0x38
    q = torch.randint(0, 4, (n, k // 2), generator=gen, device=DEV)
    q = (0x22 | (q & 1) << 3 | (q & 2) << 6).to(torch.uint8)
    xs, ws = (torch.randint(67, 188, (r, nblk), generator=gen, device=DEV) for r in (m, n))        # (2^-60 .. 2^60: any two make a BF16 number)
    xs[:, nblk // 2], ws[:, nblk // 3] = 70, 187
    sign = torch.where(q.long()[:, at // 2] >> (3 + 4 * (at % 2)) & 1 == 1, -1.0, 1.0)
    want = (sign * torch.exp2((xs[rows, at // 32][None] + ws[:, at // 32] - 254).double())).T
    assert torch.equal(want, want.to(torch.bfloat16).double())
    y = binding.mxfp4_w4a8_gemm(x8, xs.to(torch.uint8), q, ws.to(torch.uint8))
    assert torch.equal(y.double(), want)
    xs[m // 3, 0], xs[m - 1, nblk - 1], ws[0, nblk - 1], ws[n - 1, 0], ws[n // 2, nblk // 2] = 255, 255, 255, 255, 255
    x8[m // 2, k - 1] = 0xFF
    want[[m // 3, m - 1, m // 2]] = torch.nan
    want[:, [0, n - 1, n // 2]] = torch.nan
    y = binding.mxfp4_w4a8_gemm(x8, xs.to(torch.uint8), q, ws.to(torch.uint8)).double()
    assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y.nan_to_num(), want.nan_to_num())


@pytest.mark.parametrize("m,n", BLOCKS)
def test_product_in_place_of_a_strided_residual(m, n):
    k = 2272
    x8, xs = binding.mxfp4_e4m3_direct_cast(_bf16((m, k), 1))
    q, s = binding.mxfp4_direct_cast(_bf16((n, k), 2, 0.05, 4.0))
    r = _bf16((m, n), 3)
    want = binding.mxfp4_w4a8_gemm(x8, xs, q, s, residual=r)
    plain.near(want, *plain.product(x8, xs, q, s, residual=r, device=DEV))
    for extra in (3, 16 - n % 8):                               # rows at odd addresses, and where whole pieces are aligned
        held = torch.full((m, n + extra), float("nan"), dtype=torch.bfloat16, device=DEV)
        y = held[:, :n]
        y.copy_(r)
        assert binding.mxfp4_w4a8_gemm(x8, xs, q, s, residual=y, y=y) is y and torch.equal(y, want)
        assert bool(held[:, n:].isnan().all())


def test_calls_of_no_rows():
    """Nothing to do for the norm and the adapters; the product refuses it, as the other products do."""
    x, w = torch.empty((0, 64), dtype=torch.bfloat16, device=DEV), torch.ones(64, dtype=torch.bfloat16, device=DEV)
    got = binding.mxfp4_rms_norm(x, w, residual=x.clone(), out="both")
    assert got.y.shape == got.total.shape == got.q8.shape == (0, 64) and got.s.shape == (0, 2)
    a, b = torch.ones((2, 8, 64), dtype=torch.bfloat16, device=DEV), torch.ones((2, 24, 8), dtype=torch.bfloat16, device=DEV)
    assert binding.mxfp4_lora(x, a, b, torch.empty(0, dtype=torch.int32, device=DEV)).shape == (0, 24)
    q, s = binding.mxfp4_direct_cast(_bf16((8, 64), 1))
    with pytest.raises(binding.Mxfp4Error, match="M=0"):
        binding.mxfp4_w4a8_gemm(got.q8, got.s, q, s)
