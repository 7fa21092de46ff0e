"""The FP8 quantisers with block scales, the grouped product on them and the layer, on
the GPU against the float64 oracle.

Codes and scales of the quantisers must be equal.  A product in bf16 is off by half a
step of the result (2^-8) and by the float32 sums before it, whose products are exact.
Of a few rows, blocks folded into a total: 128 products in steps of four, each rounding (or
truncating) by at most 2^-23 of the block's sum of |products|, 32 * 2^-23 = 2^-18; the
product of the two scales, the fold and the total once a block, 3 * 23 * 2^-24 < 2^-17.8 at
K = 2880.  Of more, one sum over K = n products, rescaled once a block: the unit, its
reciprocal (2^-23), their product and the multiplication, 5 * 2^-24 for each of the blocks
still to come, half of 23 on average, 2^-18.1; n / 4 steps that round the sum so far by
2^-23, which for products of either sign lies within 4 standard deviations, 4 * 1.25 / sqrt(n)
of the sum of |products| at the end and half of that on average: 0.63 sqrt(n) 2^-23 < 2^-17.8.
Either stays below 2^-16.8 of the sum of |products|."""

import numpy as np
import pytest
import torch

from oracle import fp8_block as OB
from paper_2607_15810_amd import ops
from paper_2607_15810_amd import quads as Q

pytestmark = pytest.mark.gpu

DEV = "cuda"
FLOOR = 2.0 ** -16.8
HALF = 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.lib()
    yield


def np_of(t):
    return t.detach().cpu().numpy()


def bits(a):
    return np.ascontiguousarray(a, np.float32).view(np.uint32)


def up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def stream():
    return torch.cuda.current_stream().cuda_stream


# ------------------------------------------------------------------ quantisers

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 16), (1, 4096), (15, 128), (16, 144), (17, 400),
                                       (33, 512), (130, 528), (257, 2880)])
def test_quantize_act(rows, cols, dtype):
    rng = np.random.default_rng(rows + cols)
    x = rng.standard_normal((rows, cols + 8)).astype(np.float32) * 3
    x[rows // 2, :cols // 2] = 0.0
    x[rows - 1, 0] = 3e4                           # the rest of the block subnormal
    x[0, :8] *= 1e-33                              # small, and below 2^-100 with the next line
    if cols > 128:
        x[0, 128:256] = 1e-31
    wide = torch.from_numpy(x).to(DEV).to(dtype)
    v = wide[:, :cols]                             # rows cols + 8 apart
    codes, scales = ops.fp8_block_quantize_act(v)
    rc, rs = OB.quantize_act(np_of(v.float()))
    assert np.array_equal(np_of(codes), rc)
    assert np.array_equal(bits(np_of(scales)), bits(rs))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E,N,K", [(1, 16, 16), (2, 128, 128), (3, 144, 272), (2, 400, 48),
                                   (1, 8, 256), (5, 256, 384)])
def test_quantize_weight(E, N, K, dtype):
    rng = np.random.default_rng(N + K)
    w = torch.from_numpy(rng.standard_normal((E, N, K)).astype(np.float32)).to(DEV).to(dtype)
    w[0, :4] = 0
    rc, rs = OB.quantize_weight(np_of(w.float()))
    codes, scales = ops.fp8_block_quantize_weight(w)
    assert np.array_equal(np_of(codes), rc) and np.array_equal(bits(np_of(scales)), bits(rs))
    if N % 16 == 0:
        c, s, ct, st = ops.fp8_block_quantize_weight(w, transposed=True)
        assert torch.equal(c, codes) and torch.equal(s, scales)
        assert np.array_equal(np_of(ct), rc.transpose(0, 2, 1))
        assert np.array_equal(bits(np_of(st)), bits(rs.transpose(0, 2, 1)))


def test_quantise_not_finite():
    x = torch.ones((4, 256), device=DEV)
    x[0, 3] = float("nan")
    x[1, 130] = float("inf")
    x[2, 5] = -float("inf")
    codes, scales = ops.fp8_block_quantize_act(x)
    v = codes.view(torch.float8_e4m3fn).float() * scales.t().repeat_interleave(128, 1)
    want = torch.zeros((4, 256), dtype=torch.bool)
    want[0, 3] = True
    want[1, 128:] = True
    want[2, :128] = True
    assert torch.equal(torch.isnan(v).cpu(), want)
    assert (v[~want.to(DEV)] == 1.0).all()


# ------------------------------------------------------------------ products

def make(rng, counts, N, K, a_rows=None, gather=True):
    """Operands of experts with `counts` rows."""
    E, rows = len(counts), int(sum(counts))
    offs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    a_rows = a_rows or max(rows, 1)
    x = rng.standard_normal((a_rows, K)).astype(np.float32)
    x[:, :: max(1, K // 5)] *= 8.0
    a, sa = OB.quantize_act(x)
    w, sw = OB.quantize_weight(rng.standard_normal((E, N, K)).astype(np.float32) * 0.1)
    tok = rng.integers(0, a_rows, rows).astype(np.int32) if gather else None
    return a, sa, w, sw, tok, offs, rows


def refs(a, sa, w, sw, tok, offs):
    return OB.grouped_gemm(a, sa, tok, offs, w, sw)


def check_bf16(got, ref, mag):
    err = np.abs(np_of(got.float()).astype(np.float64) - ref)
    bound = HALF * np.abs(ref) + FLOOR * mag * (1 + HALF)
    assert (err <= bound).all(), f"{(err > bound).sum()} of {err.size}, worst {(err / bound).max()}"


def swiglu_ref(gu, mag):
    """silu(g) u and a bound of its error: g and u off by FLOOR of their products' sums
    (|silu'| <= 1.1), and 2^-16 relative for the exponential (an argument below 100
    times 2^-23) and the reciprocal."""
    I = gu.shape[1] // 2
    g, u = gu[:, :I], gu[:, I:]
    h = OB.silu(g) * u
    e = FLOOR * (1.1 * np.abs(u) * mag[:, :I] + np.abs(OB.silu(g)) * mag[:, I:]
                 + 1.1 * FLOOR * mag[:, :I] * mag[:, I:]) + 2.0 ** -16 * np.abs(h)
    return h, e


def check_swiglu(got, gu, mag):
    h, e = swiglu_ref(gu, mag)
    err = np.abs(np_of(got.float()).astype(np.float64) - h)
    assert (err <= HALF * np.abs(h) + e * (1 + HALF)).all()


def check_swiglu_fp8(codes, scales, gu, mag):
    h, e = swiglu_ref(gu, mag)
    rows, I = h.shape
    dec = np_of(scales).astype(np.float64)
    assert dec.shape == (-(-I // 128), rows)
    c = np_of(codes)
    val = OB.act_values(c, np_of(scales))
    for b in range(dec.shape[0]):
        s = slice(128 * b, min(I, 128 * (b + 1)))
        m, em = np.abs(h[:, s]).max(1), e[:, s].max(1)
        # 448 / m and its reciprocal: a rounding each
        assert (np.abs(dec[b] * 448 - m) <= em + m * 2.0 ** -22).all()
        # a code is within half a step of e4m3 of its value: 2^-4 of it, 2^-10 of the
        # scale below the smallest normal number
        tol = e[:, s] + (np.abs(h[:, s]) + e[:, s]) * 2.0 ** -4 * 1.001 + dec[b][:, None] * 2.0 ** -10
        assert (np.abs(val[:, s] - h[:, s]) <= tol).all()
        assert ((c[:, s] & 0x7F).max(1) == 0x7E).all()


GEMMS = [
    # counts, N, K: short and odd K, N off 32 and 128, empty experts, one row, tall ones
    ([1], 8, 16), ([5], 40, 48), ([0, 3, 0, 1], 64, 128), ([33], 264, 144),
    ([64, 1, 0, 70], 256, 256), ([200, 31], 136, 400), ([7, 9, 300], 384, 640),
    ([32, 32], 512, 2048), ([2] * 40, 320, 272), ([129, 0, 65], 192, 1168), ([513], 128, 2880),
    ([1] * 8, 1536, 2048), ([700, 20], 640, 768), ([70], 8, 16), ([90, 3], 64, 48),
    ([17, 8, 0, 9], 704, 1168), ([2, 1], 128, 7168),
    # the most experts, one row or none
    ([(e * 7 % 5 > 0) + (e % 97 == 3) for e in range(1024)], 64, 144),
    # enough workgroups or rows for the large kernel, at the same odd sizes
    ([40 * e % 97 for e in range(60)], 264, 144), ([3 * (e % 3) for e in range(200)], 136, 16),
    ([200, 31] * 20, 136, 400), ([7, 9, 300] * 30, 384, 640), ([129, 0, 65] * 16, 704, 1168),
    ([513, 700], 2560, 2880), ([64, 1, 0, 70] * 20, 256, 256), ([700, 20] * 3, 640, 768),
    # more tiles than CUs, of every height, walked from both ends
    ([37 * e % 191 for e in range(60)], 2048, 144), ([97 * e % 301 for e in range(24)], 3584, 272),
]
IDS = ["_".join(map(str, c[0][:3])) + f"e{len(c[0])}n{c[1]}k{c[2]}" for c in GEMMS]


@pytest.mark.parametrize("case", GEMMS, ids=IDS)
def test_grouped_gemm(case):
    counts, N, K = case
    rng = np.random.default_rng(N * K)
    for gather in (True, False):
        a, sa, w, sw, tok, offs, rows = make(rng, counts, N, K, a_rows=97 if gather else None,
                                             gather=gather)
        ref, mag = refs(a, sa, w, sw, tok, offs)
        args = (up(a), up(sa), up(w), up(sw), rows, up(tok) if gather else None, up(offs))
        check_bf16(ops.fp8_block_grouped_gemm(*args), ref, mag)
        if N % 64 == 0:
            check_swiglu(ops.fp8_block_grouped_gemm(*args, epilogue="swiglu"), ref, mag)
            c, s = ops.fp8_block_grouped_gemm(*args, epilogue="swiglu_quant")
            check_swiglu_fp8(c, s, ref, mag)


def test_one_matrix_without_offsets():
    rng = np.random.default_rng(9)
    a, sa, w, sw, tok, offs, rows = make(rng, [77], 192, 304, gather=False)
    ref, mag = refs(a, sa, w, sw, None, offs)
    check_bf16(ops.fp8_block_grouped_gemm(up(a), up(sa), up(w), up(sw), rows), ref, mag)


@pytest.mark.parametrize("live,rows", [(5, 8), (0, 40), (130, 300), (2600, 4000)])
@pytest.mark.parametrize("epi", [Q.QD_EPI_NONE, Q.QD_EPI_SWIGLU, Q.QD_EPI_SWIGLU_FP8])
def test_rows_behind_the_last_are_left(live, rows, epi):
    rng = np.random.default_rng(live)
    E, N, K = 4, 192, 160
    a, sa, w, sw, tok, offs, _ = make(rng, [live - live // 3, 0, live // 3, 0], N, K, a_rows=rows)
    tok = np.concatenate([tok, np.full(rows - live, -1, np.int32)])
    cols = N if epi == Q.QD_EPI_NONE else N // 2
    nb = (cols + 127) // 128
    per = 1 if epi == Q.QD_EPI_SWIGLU_FP8 else 2
    # a line before and after the outputs shows writes outside them
    out = torch.full((rows + 2, cols * per), 0x5A, dtype=torch.uint8, device=DEV)
    osc = torch.full((nb * rows + 128,), 5.0, device=DEV)
    o, s0 = out[1:], osc[64:]
    t = [up(v) for v in (a, sa, tok, offs, w, sw)]
    ws = torch.full((1 << 20,), 0xFF, dtype=torch.uint8, device=DEV)
    Q.call("moe_fp8_block_grouped_gemm", t[0].data_ptr(), t[1].data_ptr(), rows, t[2].data_ptr(),
           t[3].data_ptr(), E, rows, t[4].data_ptr(), t[5].data_ptr(), N, K, epi, o.data_ptr(),
           s0.data_ptr(), ws.data_ptr(), ws.numel(), stream())
    assert (out[0] == 0x5A).all() and (out[1 + live:] == 0x5A).all()
    assert (osc[:64] == 5.0).all() and (osc[64 + nb * rows:] == 5.0).all()
    sc = osc[64:64 + nb * rows].view(nb, rows)
    assert (sc[:, live:] == 5.0).all()
    ref, mag = refs(a, sa, w, sw, tok[:live], offs)
    o = o[:live]
    if epi == Q.QD_EPI_NONE:
        check_bf16(o.contiguous().view(torch.bfloat16), ref, mag)
    elif epi == Q.QD_EPI_SWIGLU:
        check_swiglu(o.contiguous().view(torch.bfloat16), ref, mag)
    elif live:
        check_swiglu_fp8(o, sc[:, :live].contiguous(), ref, mag)


def test_scales_reach_their_blocks():
    """One-hot operands: v[r][n] is exactly the two scales' product."""
    N, K = 264, 400
    a = np.zeros((4, K), np.uint8)
    w = np.zeros((1, N, K), np.uint8)
    one = 0x38                                    # 1.0
    for r in range(4):
        a[r, 128 * r + 5 if r < 3 else K - 1] = one
    w[0, :, [5, 133, 261, K - 1]] = one
    sa = (2.0 ** np.arange(16).reshape(4, 4)).astype(np.float32)
    sw = (2.0 ** -np.arange(12).reshape(1, 3, 4)).astype(np.float32)
    y = np_of(ops.fp8_block_grouped_gemm(up(a), up(sa), up(w), up(sw), 4).float())
    for r in range(4):
        for n in range(N):
            assert y[r, n] == sa[r, r] * sw[0, n // 128, r]


@pytest.mark.parametrize("rows", [3, 200, 6000])
def test_scales_of_all_sizes(rows):
    """Scales over 2^-60 .. 2^40, of either sign: a block's products under those of others."""
    rng = np.random.default_rng(rows)
    N, K = 192, 1040
    a, sa, w, sw, _, offs, _ = make(rng, [rows], N, K, gather=False)
    sa = (sa * 2.0 ** rng.integers(-50, 30, sa.shape) * rng.choice([-1, 1], sa.shape)).astype(np.float32)
    sw = (sw * 2.0 ** rng.integers(-10, 10, sw.shape) * rng.choice([-1, 1], sw.shape)).astype(np.float32)
    ref, mag = refs(a, sa, w, sw, None, offs)
    check_bf16(ops.fp8_block_grouped_gemm(up(a), up(sa), up(w), up(sw), rows), ref, mag)


@pytest.mark.parametrize("rows", [3, 200, 6000])
def test_scales_of_the_largest_and_smallest_sizes(rows):
    """Rows of scales near 2^-125 and near 2^117 against weights of the opposite."""
    rng = np.random.default_rng(rows)
    N, K = 192, 528
    for e in (-125, 117):
        a, sa, w, sw, _, offs, _ = make(rng, [rows], N, K, gather=False)
        sa = rng.uniform(1, 2, sa.shape).astype(np.float32) * np.float32(2.0 ** e)
        sw = rng.uniform(1, 2, sw.shape).astype(np.float32) * np.float32(2.0 ** (-e - 8))
        ref, mag = refs(a, sa, w, sw, None, offs)
        check_bf16(ops.fp8_block_grouped_gemm(up(a), up(sa), up(w), up(sw), rows), ref, mag)


@pytest.mark.parametrize("rows", [3, 200, 6000])
@pytest.mark.parametrize("ea,ew", [(-73, -73), (-109, -37), (-37, -109)])
def test_products_of_small_scales(rows, ea, ew):
    """Scales whose product is far below float32's normal numbers under sums that lift the
    results to them: bf16's steps are 2^-133 from 2^-126 down, and float32 sums that are
    subnormal round by 2^-150 a product more (K = 528: less than 2^-140 together)."""
    rng = np.random.default_rng(rows)
    N, K = 192, 528
    a, sa, w, sw, _, offs, _ = make(rng, [rows], N, K, gather=False)
    sa = rng.uniform(1, 2, sa.shape).astype(np.float32) * np.float32(2.0 ** ea)
    sw = rng.uniform(1, 2, sw.shape).astype(np.float32) * np.float32(2.0 ** ew)
    ref, mag = refs(a, sa, w, sw, None, offs)
    assert (np.abs(ref) > 2.0 ** -127).mean() > 0.25
    y = ops.fp8_block_grouped_gemm(up(a), up(sa), up(w), up(sw), rows)
    err = np.abs(np_of(y.float()).astype(np.float64) - ref)
    bound = HALF * np.abs(ref) + FLOOR * mag * (1 + HALF) + 2.0 ** -134 + 2.0 ** -140
    assert (err <= bound).all(), f"{(err > bound).sum()} of {err.size}, worst {(err / bound).max()}"


@pytest.mark.parametrize("rows", [3, 200, 6000])
def test_products_of_large_scales(rows):
    """Two scales whose product no float32 holds: over products that are all zero they add
    nothing, over small ones what those make."""
    rng = np.random.default_rng(rows)
    N, K = 192, 528
    a, sa, w, sw, _, offs, _ = make(rng, [rows], N, K, gather=False)
    a[:, 128:256] &= 0x80                          # zeros of either sign
    a[:, 256:384] = 0x01 | (a[:, 256:384] & 0x80)  # 2^-9, against weights of 2^-9
    w[:, :, 256:384] = 0x01 | (w[:, :, 256:384] & 0x80)
    ref, mag = refs(a, sa, w, sw, None, offs)
    sa[1], sw[:, :, 1] = np.float32(2.0 ** 70), np.float32(1.5 * 2.0 ** 75)
    y = ops.fp8_block_grouped_gemm(up(a), up(sa), up(w), up(sw), rows)
    check_bf16(y, ref, mag)
    sa[2], sw[:, :, 2] = np.float32(1.5 * 2.0 ** 66), np.float32(1.25 * 2.0 ** 66)
    ref, mag = refs(a, sa, w, sw, None, offs)
    check_bf16(ops.fp8_block_grouped_gemm(up(a), up(sa), up(w), up(sw), rows), ref, mag)


@pytest.mark.parametrize("rows", [3, 200, 6000])
def test_an_infinite_scale_makes_nan(rows):
    rng = np.random.default_rng(rows)
    N, K = 256, 400
    a, sa, w, sw, _, offs, _ = make(rng, [rows], N, K, gather=False)
    for bad in (float("inf"), -float("inf"), float("nan")):
        s, v = up(sa), up(sw)
        s[2, 0] = bad
        assert torch.isnan(ops.fp8_block_grouped_gemm(up(a), s, up(w), v, rows)[0]).all()
        s, v[0, 1, 2] = up(sa), bad
        y = ops.fp8_block_grouped_gemm(up(a), s, up(w), v, rows)
        assert torch.isnan(y[:, 128:]).all() and torch.isfinite(y[:, :128]).all()


@pytest.mark.parametrize("rows", [3, 200, 6000])
def test_scales_of_zero_and_not_finite(rows):
    rng = np.random.default_rng(rows)
    N, K = 256, 400
    a, sa, w, sw, _, offs, _ = make(rng, [rows], N, K, gather=False)
    sa[1, 1] = 0.0                                 # a block that stands for zeros
    ref, mag = refs(a, sa, w, sw, None, offs)
    args = [up(a), up(sa), up(w), up(sw), rows]
    check_bf16(ops.fp8_block_grouped_gemm(*args), ref, mag)
    clean = ops.fp8_block_grouped_gemm(*args)
    for bad in (float("nan"), float("inf")):
        args[1][2, 0] = bad
        y = ops.fp8_block_grouped_gemm(*args)
        assert not torch.isfinite(y[0]).any() and torch.equal(y[1:], clean[1:])
    args[1] = up(sa)
    args[3][0, 1, 2] = float("nan")                # columns 128 .. 255
    y = ops.fp8_block_grouped_gemm(*args)
    assert torch.isnan(y[:, 128:]).all() and torch.equal(y[:, :128], clean[:, :128])


def test_offsets_past_32_bits():
    """Weights of 5 GiB (each expert below 4), an output of 5 GB, activations of 4.6 GB."""
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    E, N, K = 5, 16384, 65536
    w = torch.randint(0, 0x7F, (E, N, K), dtype=torch.uint8, generator=g, device=DEV)
    sw = torch.rand((E, N // 128, K // 128), generator=g, device=DEV) + 0.5
    a = torch.randint(0, 0x7F, (6, K), dtype=torch.uint8, generator=g, device=DEV)
    sa = torch.rand((K // 128, 6), generator=g, device=DEV) + 0.5
    offs = torch.tensor([0, 1, 2, 3, 3, 6], dtype=torch.int32, device=DEV)
    y = ops.fp8_block_grouped_gemm(a, sa, w, sw, 6, None, offs)
    one = ops.fp8_block_grouped_gemm(a[3:].contiguous(), sa[:, 3:].contiguous(), w[4:].contiguous(),
                                     sw[4:].contiguous(), 3)
    # the call of one expert may run on the other kernel, whose sums have another order:
    # every product is positive, so each result is within HALF + FLOOR of the exact sum
    assert ((y[3:].double() - one.double()).abs() <= 2.1 * (HALF + FLOOR) * one.double()).all()
    del w
    rows, N, K = 1 << 20, 2560, 16
    a = torch.randint(0, 0x7F, (rows, K), dtype=torch.uint8, generator=g, device=DEV)
    sa = torch.rand((1, rows), generator=g, device=DEV)
    w = torch.randint(0, 0x7F, (1, N, K), dtype=torch.uint8, generator=g, device=DEV)
    sw = torch.rand((1, N // 128, 1), generator=g, device=DEV)
    y = ops.fp8_block_grouped_gemm(a, sa, w, sw, rows)
    last = ops.fp8_block_grouped_gemm(a[-300:].contiguous(), sa[:, -300:].contiguous(), w, sw, 300)
    assert torch.equal(y[-300:], last)
    del y, a
    # k rows of each token: more than 4 GiB of codes if they were not gathered
    rows, K = 140000, 32768
    a = torch.randint(0, 0x7F, (7, K), dtype=torch.uint8, generator=g, device=DEV)
    sa = torch.rand((K // 128, 7), generator=g, device=DEV)
    w = torch.randint(0, 0x7F, (1, 64, K), dtype=torch.uint8, generator=g, device=DEV)
    sw = torch.rand((1, 1, K // 128), generator=g, device=DEV)
    tok = (torch.arange(rows, device=DEV) % 7).int()
    y = ops.fp8_block_grouped_gemm(a, sa, w, sw, rows, tok)
    assert torch.equal(y, y[:7].repeat(20000, 1))
    del y, tok
    x = torch.randn((70016, 65536), dtype=torch.bfloat16, generator=g, device=DEV)
    codes, scales = ops.fp8_block_quantize_act(x)
    c, s = ops.fp8_block_quantize_act(x[-40:])
    assert torch.equal(codes[-40:], c) and torch.equal(scales[:, -40:], s)


# (the first two on the large kernel, the last on that of few rows)
@pytest.mark.parametrize("rows,N,K", [(1400, 2560, 7168), (1400, 2560, 2816), (9, 256, 7168)])
def test_long_sums_do_not_drift(rows, N, K):
    """The second half of K takes off what the first has summed: 0 to the exact sum, so what is
    left is the rounding.  Codes of 1/4 to 4: the products of a half are multiples of 2^-10
    whose sums stay below 2^14, so the float32 sums of one unit are exact.  The large kernel's
    are then 0 where all blocks have the same scales.  Of others, a block is rescaled K / 128
    times at most by a quotient and a product, 2^-24 each, its unit is a product rounded
    once: (K / 128 + 1) 2^-23 of the sum of |products|.  The few-rows kernel folds a block with
    two roundings of the total, and joins four: as many."""
    g = torch.Generator(device=DEV)
    g.manual_seed(K)
    half = lambda *n: torch.randint(0x28, 0x49, n, dtype=torch.uint8, generator=g, device=DEV)
    a, w = half(rows, K // 2), half(1, N, K // 2)
    a, w = torch.cat([a, a ^ 0x80], 1), torch.cat([w, w], 2)
    blocks, nb = K // 256, N // 128
    v = lambda c: c.view(torch.float8_e4m3fn).float()
    assert float((v(a[:, :K // 2]) @ v(w[0, :, :K // 2]).t()).max()) < 2 ** 14
    for ma, mw in ((1.3, 1.7), (1.0, 1.37), (1.9, 1.1), (1.5, 1.25), (1.77, 1.61)):
        sa = torch.full((2 * blocks, rows), ma, device=DEV)
        sw = torch.full((1, nb, 2 * blocks), mw, device=DEV)
        y = ops.fp8_block_grouped_gemm(a, sa, w, sw, rows)
        if rows > 9:
            assert not y.any()
    sa = torch.rand((blocks, rows), generator=g, device=DEV) + 0.5
    sw = torch.rand((1, nb, blocks), generator=g, device=DEV) + 0.5
    sa, sw = torch.cat([sa, sa]), torch.cat([sw, sw], 2)
    y = ops.fp8_block_grouped_gemm(a, sa, w, sw, rows)
    wide = lambda s, n: s.repeat_interleave(128, 0)[:n].double()
    mag = (v(a).abs().double() * wide(sa, K).t()) @ (
        v(w[0]).double() * wide(sw[0].t().contiguous(), K).t().repeat_interleave(128, 0)[:N]).t()
    assert (y.double().abs() <= mag * (K / 128 + 1) * 2.0 ** -23 * (1 + HALF)).all()


@pytest.mark.parametrize("counts,N,K", [([700, 650], 2560, 7168), ([1300], 2560, 20480)])
def test_long_k_on_the_large_kernel(counts, N, K):
    """Against the oracle: half a bf16 step, (K / 128 + 1) 2^-23 of rescaling and the rounding of
    K / 4 steps of the sum so far, 0.63 sqrt(K) 2^-23 of the sum of |products|."""
    rng = np.random.default_rng(K)
    a, sa, w, sw, tok, offs, rows = make(rng, counts, N, K, a_rows=60)
    assert Q.lib().moe_fp8_block_grouped_gemm_workspace(rows, N, K, len(counts), Q.QD_EPI_SWIGLU_FP8) == 0
    ref, mag = refs(a, sa, w, sw, tok, offs)
    y = ops.fp8_block_grouped_gemm(up(a), up(sa), up(w), up(sw), rows, up(tok), up(offs))
    err = np.abs(np_of(y.float()).astype(np.float64) - ref)
    floor = (K / 128 + 1 + 0.63 * K ** 0.5) * 2.0 ** -23
    assert (err <= HALF * np.abs(ref) + floor * mag * (1 + HALF)).all()


def random_codes(E, N, K, rows, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    code = lambda *n: torch.randint(0, 256, n, dtype=torch.uint8, generator=g, device=DEV) & 0xF7
    scale = lambda *n: torch.rand(n, generator=g, device=DEV) + 0.5
    return (code(rows, K), scale(-(-K // 128), rows), code(E, N, K),
            scale(E, -(-N // 128), -(-K // 128)))


# (the large kernel, in every tile height; the other, in both of its)
@pytest.mark.parametrize("N,K,calls", [
    (16384, 1040, [(300, 200), (700, 130), (131, 0)]), (16384, 4096, [(300, 200), (131, 0)]),
    (256, 1040, [(1, 0), (3, 2), (40, 0), (131, 60)])])
def test_a_row_does_not_depend_on_the_batch(N, K, calls):
    """The bits of a row are the same in every tile height, at any place and beside any
    other rows."""
    t = random_codes(2, N, K, 900, 8)
    first, rest = (700, 200) if N > 256 else (150, 60)
    place = np.concatenate([np.arange(first), 700 + np.arange(rest)]).astype(np.int32)
    whole = ops.fp8_block_grouped_gemm(*t, first + rest, up(place),
                                       up(np.array([0, first, first + rest], np.int32)))
    for n0, n1 in calls:
        at = np.concatenate([np.arange(n0)[::-1], first + np.arange(n1)])
        y = ops.fp8_block_grouped_gemm(*t, n0 + n1, up(place[at]),
                                       up(np.array([0, n0, n0 + n1], np.int32)))
        assert torch.equal(y, whole[up(at)])


@pytest.mark.parametrize("counts", [[5, 2], [40, 30], [4000, 3000]])
def test_a_nan_row_stays_alone(counts):
    rng = np.random.default_rng(4)
    a, sa, w, sw, tok, offs, rows = make(rng, counts, 256, 256, gather=False)
    args = [up(a), up(sa), up(w), up(sw), rows, None, up(offs)]
    clean = ops.fp8_block_grouped_gemm(*args)
    args[0][4, 100] = 0x7F
    y = ops.fp8_block_grouped_gemm(*args)
    keep = [r for r in range(rows) if r != 4]
    assert torch.isnan(y[4]).all() and torch.equal(y[keep], clean[keep])


def test_input_gradient():
    """dx = dy w through the transposed bank, against the formula and against
    differences of <dy, x w^T> (linear in x: exact up to rounding)."""
    rng = np.random.default_rng(12)
    counts, N, K = [20, 0, 45], 144, 272
    offs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rows = int(offs[-1])
    w = up(rng.standard_normal((3, N, K)).astype(np.float32))
    c, s, ct, st = ops.fp8_block_quantize_weight(w, transposed=True)
    dy = up(rng.standard_normal((rows, N)).astype(np.float32))
    qc, qs = ops.fp8_block_quantize_act(dy)
    dx = ops.fp8_block_grouped_gemm(qc, qs, ct, st, rows, None, up(offs))
    v, wv = OB.act_values(np_of(qc), np_of(qs)), OB.weight_values(np_of(c), np_of(s))
    ref, mag = np.zeros((rows, K)), np.zeros((rows, K))
    for e in range(3):
        r = slice(offs[e], offs[e + 1])
        ref[r], mag[r] = v[r] @ wv[e], np.abs(v[r]) @ np.abs(wv[e])
    check_bf16(dx, ref, mag)
    x = rng.standard_normal((rows, K))
    loss = lambda x: sum((v[r] * (x[r] @ wv[e].T)).sum() for e, r in enumerate(
        slice(offs[e], offs[e + 1]) for e in range(3)))
    for i, j in [(0, 0), (19, 271), (20, 5), (64, 128)]:
        d = np.zeros_like(x)
        d[i, j] = 1.0
        diff = (loss(x + d) - loss(x - d)) / 2
        assert abs(float(dx[i, j]) - diff) <= HALF * abs(diff) + FLOOR * mag[i, j] * 1.01 + 1e-9


# ------------------------------------------------------------------ the layer

def layer_inputs(T, H, I, E, seed):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((T, H)).astype(np.float32)).to(DEV).to(torch.bfloat16)
    lg = up(rng.standard_normal((T, E)).astype(np.float32))
    w13 = up(rng.standard_normal((E, 2 * I, H)).astype(np.float32) * 0.05)
    w2 = up(rng.standard_normal((E, H, I)).astype(np.float32) * 0.05)
    return (x, lg, ops.fp8_block_quantize_weight(w13), ops.fp8_block_quantize_weight(w2),
            up((0.2 * rng.standard_normal(E)).astype(np.float32)))


LAYERS = [
    (1, 64, 32, 4, 2, dict()), (1, 2048, 768, 16, 8, dict(scoring="sigmoid", groups=4, top_groups=2)),
    (7, 272, 96, 8, 3, dict(scoring="sigmoid", bias=True, scale=2.5)),
    (64, 256, 160, 8, 2, dict(renorm=False)), (130, 400, 128, 6, 4, dict(bias=True)),
    (500, 512, 256, 4, 2, dict(scoring="sigmoid", bias=True, groups=2, top_groups=1)),
    (300, 1024, 384, 32, 8, dict(bias=True, groups=8, top_groups=4, group_sum=2)),
    (2000, 512, 256, 16, 4, dict(bias=True)), (1500, 400, 96, 6, 4, dict(scoring="sigmoid")),
]


@pytest.mark.parametrize("live", [False, True])
@pytest.mark.parametrize("case", LAYERS, ids=[f"t{c[0]}_h{c[1]}_i{c[2]}" for c in LAYERS])
def test_layer(case, live):
    T, H, I, E, k, kw = case
    kw = dict(kw)
    x, lg, w13, w2, b = layer_inputs(T, H, I, E, T + H)
    if kw.pop("bias", False):
        kw["bias"] = b
    lv = None
    if live:
        lv = torch.from_numpy(np.random.default_rng(T).random(T) < 0.7).to(DEV)
        lv[T // 2] = False
    lay = ops.FP8BlockMoELayer(*w13, *w2, T, k, **kw)
    y = lay(x, lg, live=lv)
    # its calls one after the other: the same bits
    ids, w, offs, tok, inv = ops.route_scored(lg, k, live=lv, **kw)
    R = T * k
    h = ops.fp8_block_grouped_gemm(*ops.fp8_block_quantize_act(x), *w13, R, tok, offs,
                                   epilogue="swiglu_quant")
    z = ops.fp8_block_grouped_gemm(*h, *w2, R, None, offs)
    assert torch.equal(y, ops.unpermute_combine(z, inv, w))
    if lv is not None:
        assert not y[~lv].any()
    # free-running against the oracle: an error of h moves a code of it by a step now
    # and then, as in the other FP8 layer's tests
    okw = dict(kw, bias=np_of(b)) if "bias" in kw else kw
    ref = OB.moe_layer(np_of(x.float()), np_of(lg), tuple(map(np_of, w13)), tuple(map(np_of, w2)), k,
                       live=None if lv is None else np_of(lv), **okw)
    got = np_of(y.float()).astype(np.float64)
    n = np.linalg.norm(ref["y"])
    assert np.linalg.norm(got - ref["y"]) <= 1e-2 * (n if n else 1.0)


def test_layer_every_token_dead_over_stale_memory():
    x, lg, w13, w2, _ = layer_inputs(9, 128, 64, 4, 3)
    lay = ops.FP8BlockMoELayer(*w13, *w2, 9, 2)
    lay.ws.fill_(0xFF)                             # NaN wherever a result is not written
    y = lay(x, lg, live=torch.zeros(9, dtype=torch.uint8, device=DEV))
    assert not y.any()


def test_layer_no_tokens():
    x, lg, w13, w2, _ = layer_inputs(3, 128, 64, 4, 3)
    lay = ops.FP8BlockMoELayer(*w13, *w2, 0, 2)
    assert lay(x[:0].contiguous(), lg[:0].contiguous()).shape == (0, 128)


def test_layers_captured_and_on_another_stream():
    T, k = 48, 4
    x, lg, w13, w2, b = layer_inputs(T, 512, 192, 16, 5)
    x2, lg2 = x.flip(0).contiguous(), lg.flip(0).contiguous()
    kw = dict(scoring="sigmoid", bias=b, groups=4, top_groups=2)
    one, two = [ops.FP8BlockMoELayer(*w13, *w2, T, k, **kw) for _ in range(2)]
    want, want2 = one(x, lg).clone(), one(x2, lg2).clone()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        other = two(x2, lg2)
    same = one(x, lg)
    torch.cuda.synchronize()
    assert torch.equal(same, want) and torch.equal(other, want2)
    xs, ls = x.clone(), lg.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = one(xs, ls)
    for p, q, w in ((x2, lg2, want2), (x, lg, want), (x2, lg2, want2)):
        xs.copy_(p)
        ls.copy_(q)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, w)
        assert torch.equal(two(p, q), w)


def test_combine_skips_slots_without_a_row():
    z = torch.full((4, 16), float("nan"), dtype=torch.bfloat16, device=DEV)
    z[1], z[2] = 2.0, 3.0
    inv = torch.tensor([[1, -1], [-1, -1], [2, 1]], dtype=torch.int32, device=DEV)
    w = torch.tensor([[0.5, 1.0], [1.0, 1.0], [1.0, 2.0]], device=DEV)
    y = ops.unpermute_combine(z, inv, w)
    assert (y[0] == 1.0).all() and (y[1] == 0.0).all() and (y[2] == 7.0).all()


@pytest.mark.parametrize("rows", [3, 200, 6000])
def test_products_of_the_largest_numbers(rows):
    """What the quantisers make of the types' largest numbers (scales to 2^119.2) is multiplied
    like any other, on either side."""
    rng = np.random.default_rng(rows)
    N, K = 192, 528
    top = float(torch.finfo(torch.bfloat16).max)
    for side in range(2):
        x = rng.standard_normal((rows, K)).astype(np.float32)
        w = rng.standard_normal((1, N, K)).astype(np.float32)
        big, small = (x, w) if side == 0 else (w, x)
        big /= np.abs(big).max()
        big[..., ::3] = np.sign(big[..., ::3])
        small *= np.float32(1e-30)
        t = torch.from_numpy(big).to(DEV) * top
        a = ops.fp8_block_quantize_act(t.to(torch.bfloat16) if side == 0 else up(small))
        b = ops.fp8_block_quantize_weight(t.to(torch.bfloat16) if side == 1 else up(small))
        assert float((a if side == 0 else b)[1].max()) > 2.0 ** 119
        ref, mag = refs(*map(np_of, a), *map(np_of, b), None, np.array([0, rows]))
        check_bf16(ops.fp8_block_grouped_gemm(*a, *b, rows), ref, mag)


@pytest.mark.parametrize("counts", [[5, 2], [40, 30], [4000, 3000]])
def test_nan_and_overflow_through_the_epilogues(counts):
    """A NaN row of h is NaN codes under a scale of 1; an h past float32 makes its block NaN
    (an infinite scale); the other rows keep their bits."""
    rng = np.random.default_rng(14)
    N, K = 512, 272
    a, sa, w, sw, tok, offs, rows = make(rng, counts, N, K, gather=False)
    args = [up(a), up(sa), up(w), up(sw), rows, None, up(offs)]
    run = lambda e: ops.fp8_block_grouped_gemm(*args, epilogue=e)
    y, (c, s) = run("swiglu"), run("swiglu_quant")
    args[0][4, 100] = 0x7F
    args[1][:, 1] = 2.0 ** 110                     # g u of about 2^230
    y2, (c2, s2) = run("swiglu"), run("swiglu_quant")
    keep = [r for r in range(rows) if r not in (1, 4)]
    assert torch.equal(y2[keep], y[keep]) and torch.equal(c2[keep], c[keep])
    assert torch.equal(s2[:, keep], s[:, keep])
    assert torch.isnan(y2[4]).all() and ((c2[4] & 0x7F) == 0x7F).all() and (s2[:, 4] == 1).all()
    assert torch.isinf(y2[1]).any() and torch.isinf(s2[:, 1]).all()
    v = c2[1].view(torch.float8_e4m3fn).float() * s2[:, 1].repeat_interleave(128)
    assert torch.isnan(v).all()
