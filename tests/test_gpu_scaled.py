"""8-bit block-scaled matrices on the GPU: ee_quantize_blocks and ee_scaled_matmul
against the fp64 oracle.

Quantising is defined down to the bit (fp32 division, reciprocal and product, then
one rounding), so codes and scales must be equal to the oracle's.

A product's terms are exact in fp32 (4 + 4 significant bits) and a block's scale
product is one rounding; every fp32 addition, in whatever order and even if a
matrix core truncates, is off by at most 2^-23 of a partial sum, which is at most
the sum of the terms' magnitudes.  With 128 additions in a block and one per block
after it (and its scaling, two roundings of 2^-24):
    |error| <= (128 + blocks + 1) 2^-23 sum |terms|,
For a bf16 C the 8-bit matrix instruction cuts each product to a multiple of 2^-13
of the power of two under the largest of its group, k / 8 (measured: 65536 beside 8
to 15 adds 8, beside 7 nothing, whichever the signs and places), so seven of eight
are off by less than 2^-13 of that largest one:
    |error| <= the above + 7 2^-13 sum over groups of max |term| + 2^-8 |result|,
the last for the rounding to bf16 (half a step).
"""

import ctypes

import numpy as np
import pytest
import torch

from oracle import scaled as Q
from paper_2402_00518_amd import binding as B

pytestmark = pytest.mark.gpu

CODES = {"e4m3": (B.EE_E4M3, torch.float8_e4m3fn), "e5m2": (B.EE_E5M2, torch.float8_e5m2)}
DTYPES = {"f32": (B.EE_F32, torch.float32), "bf16": (B.EE_BF16, torch.bfloat16)}


def stream():
    return torch.cuda.current_stream().cuda_stream


def say(msg):
    print(msg, flush=True)


def matrix(rows, cols, seed, row_scale=True):
    g = np.random.default_rng(seed)
    x = g.standard_normal((rows, cols))
    if row_scale:
        x *= np.exp(g.standard_normal((rows, 1)))
    return x.astype(np.float32)


def pad16(n):
    return -(-n // 16) * 16


class Device:
    """Codes and scales on the GPU, with spare columns and scales (ld, scale_ld larger than needed) full of marks."""

    def __init__(self, rows, cols, block_rows, code, spare=0):
        self.rows, self.cols, self.block_rows, self.code = rows, cols, block_rows, code
        self.data = torch.full((rows + (2 if spare else 0), pad16(cols) + spare), 0x7F, dtype=torch.uint8, device="cuda")
        self.scale = torch.full((-(-cols // 128), -(-rows // block_rows) + spare // 16), -1.0, device="cuda")
        self.c = B.make_scaled(self.data, self.scale, block_rows, CODES[code][0], rows=rows, cols=cols)

    @classmethod
    def of(cls, codes, scale, block_rows, code, spare=0):
        d = cls(*codes.shape, block_rows, code, spare)
        bits = torch.from_numpy(Q.encode(codes, code)).cuda()
        d.data[:d.rows, :d.cols] = bits
        d.data[:d.rows, d.cols:pad16(d.cols)] = 0
        d.scale[:, :scale.shape[1]] = torch.from_numpy(scale).cuda()
        return d


QUANT = [
    # rows, cols, dtype, block rows, code, code of the transpose, spare columns
    (1, 1, "f32", 1, "e4m3", "e4m3", 0),
    (1, 4096, "bf16", 1, "e4m3", "e4m3", 0),
    (8, 129, "bf16", 1, "e4m3", "e5m2", 16),
    (127, 65, "f32", 1, "e5m2", "e4m3", 0),
    (128, 128, "bf16", 128, "e4m3", "e4m3", 32),
    (129, 257, "f32", 128, "e4m3", "e5m2", 16),
    (300, 1000, "bf16", 128, "e5m2", "e5m2", 0),
    (777, 333, "bf16", 1, "e4m3", "e4m3", 48),
    (33, 17, "f32", 1, "e4m3", "e4m3", 16),
]


@pytest.mark.parametrize("out", ["q", "qt", "both"])
@pytest.mark.parametrize("rows,cols,dtype,br,code,code_t,spare", QUANT)
def test_codes_and_scales_are_the_oracle_s(rows, cols, dtype, br, code, code_t, spare, out):
    say(f"case: quantize {rows}x{cols} {dtype} block rows {br} {code}/{code_t} spare {spare} {out}")
    ldx = cols + (3 if spare == 16 else spare)      # (an odd stride too)
    full = torch.from_numpy(matrix(rows, ldx, rows + cols)).to("cuda").to(DTYPES[dtype][1])
    x = full[:, :cols]
    ref = x.float().cpu().numpy()
    q = Device(rows, cols, br, code, spare) if out != "qt" else None
    qt = Device(cols, rows, br, code_t, spare) if out != "q" else None
    B.ee_quantize_blocks(full, DTYPES[dtype][0], rows, cols, ldx, q and q.c, qt and qt.c, stream())
    torch.cuda.synchronize()
    for d, a in ((q, ref), (qt, ref.T)):
        if d is None:
            continue
        codes, scale = Q.quantize(np.ascontiguousarray(a), br, d.code)
        got = d.data.cpu().numpy()
        np.testing.assert_array_equal(Q.decode(got[:d.rows, :d.cols], d.code), codes)
        assert (got[:d.rows, d.cols:pad16(d.cols)] == 0).all()
        assert (got[:d.rows, pad16(d.cols):] == 0x7F).all() and (got[d.rows:] == 0x7F).all()
        s = d.scale.cpu().numpy()
        np.testing.assert_array_equal(s[:, :scale.shape[1]], scale)
        assert (s[:, scale.shape[1]:] == -1).all()


def test_extreme_values():
    x = np.zeros((6, 256), dtype=np.float32)
    x[0, :3] = [3e38, -1e38, 1e-30]
    x[1, :3] = [1e-40, -2e-41, 0.0]               # subnormal: the least scale
    x[2, 5] = np.inf
    x[3, 7], x[3, 8] = np.nan, 2.0
    x[4, 130] = -0.0
    d = Device(6, 256, 1, "e4m3")
    B.ee_quantize_blocks(torch.from_numpy(x).cuda(), B.EE_F32, 6, 256, 256, d.c, None, stream())
    v = d.data.view(torch.float8_e4m3fn).float().cpu().numpy()
    s = d.scale.cpu().numpy()
    codes, scale = Q.quantize(x[[0, 1, 4, 5]], 1, "e4m3")
    np.testing.assert_array_equal(v[[0, 1, 4, 5]], codes)
    np.testing.assert_array_equal(s[:, [0, 1, 4, 5]], scale)
    assert np.isinf(s[0, 2]) and np.isnan(v[2, 5])
    assert np.isnan(v[3, 7]) and v[3, 8] == 448 and s[0, 3] == np.float32(2.0 / 448)


def operands(m, n, k, ca, bra, brb, seed):
    a, sa = Q.quantize(matrix(m, k, seed), bra, ca)
    b, sb = Q.quantize(matrix(n, k, seed + 1, False) * np.float32(0.02), brb, "e4m3")
    return a, sa, b, sb


def reference(a, sa, bra, b, sb, brb):
    c, mag = Q.matmul(Q.values(a, sa, bra), Q.values(b, sb, brb))
    blocks = sa.shape[0]
    return c, (128 + blocks + 1) * 2.0 ** -23 * mag


def group_maxima(a, b):
    """sum over groups of eight columns of max |a_k b_k|, for every pair of rows."""
    a, b = (torch.from_numpy(np.abs(np.pad(v, ((0, 0), (0, -v.shape[1] % 8)))).astype(np.float32)).cuda() for v in (a, b))
    s = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device="cuda")
    for k in range(0, a.shape[1], 8):
        m = a[:, None, k] * b[None, :, k]
        for e in range(1, 8):
            m = torch.maximum(m, a[:, None, k + e] * b[None, :, k + e])
        s += m
    return s.cpu().numpy() * (1 + 2.0 ** -22)


MATMUL = [
    # rows of a, rows of b, depth, code of a, block rows of a and b
    (1, 1, 1, "e4m3", 1, 128),
    (1, 128, 16, "e4m3", 1, 128),
    (1, 1000, 4096, "e4m3", 1, 128),
    (2, 333, 130, "e4m3", 1, 128),
    (8, 1003, 1024, "e4m3", 1, 128),
    (16, 129, 144, "e4m3", 1, 128),
    (17, 257, 127, "e5m2", 1, 128),
    (31, 64, 2000, "e4m3", 1, 1),
    (33, 700, 1111, "e4m3", 1, 128),
    (48, 5120, 3456, "e4m3", 1, 128),
    (64, 127, 640, "e4m3", 128, 128),
    (65, 1000, 512, "e5m2", 1, 1),
    (100, 2000, 300, "e4m3", 1, 128),
    (130, 130, 128, "e4m3", 1, 128),
    (200, 515, 2048, "e4m3", 128, 1),
    (257, 1024, 1000, "e4m3", 1, 128),
    (300, 300, 4016, "e5m2", 1, 1),
    (513, 2050, 96, "e4m3", 1, 128),
    (1025, 1300, 777, "e5m2", 1, 1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k,ca,bra,brb", MATMUL)
def test_product(m, n, k, ca, bra, brb, dtype):
    say(f"case: scaled matmul {m}x{n}x{k} {ca} blocks {bra}/{brb} {dtype}")
    a, sa, b, sb = operands(m, n, k, ca, bra, brb, m + n + k)
    ref, bound = reference(a, sa, bra, b, sb, brb)
    if dtype == "bf16":
        bound = bound + 7 * 2.0 ** -13 * group_maxima(Q.values(a, sa, bra), Q.values(b, sb, brb))
        bound = bound + 2.0 ** -8 * (np.abs(ref) + bound)
    da, db = Device.of(a, sa, bra, ca), Device.of(b, sb, brb, "e4m3")
    c = torch.full((m + 1, n), 7.0, dtype=DTYPES[dtype][1], device="cuda")
    for _ in range(2):
        B.ee_scaled_matmul(da.c, db.c, c, DTYPES[dtype][0], n, 0, stream())
    got = c.double().cpu().numpy()
    err = np.abs(got[:m] - ref)
    assert (err <= bound).all(), (np.argmax(err - bound), err.max(), bound.min())
    assert (got[m] == 7).all()


def tile_of(f32, row_scales, n, m, k):
    """The tile that the library's rule gives a product (an index, see launch.h)."""
    f = ctypes.CDLL(B.LIB_PATH)["_ZN2ee11scaled_tileEbbiii"]
    f.restype, f.argtypes = ctypes.c_int, (ctypes.c_bool,) * 2 + (ctypes.c_int,) * 3
    return f(f32, row_scales, n, m, k)


def check_product(m, n, k, ca, brb, dtype, spare=0):
    a, sa, b, sb = operands(m, n, k, ca, 1, brb, m + n)
    va, vb = (torch.from_numpy(v).cuda() for v in (Q.values(a, sa, 1), Q.values(b, sb, brb)))
    ref, bound = va @ vb.t(), (129 + sa.shape[0]) * 2.0 ** -23 * (va.abs() @ vb.abs().t())
    if dtype == "bf16":
        bound = bound + 7 * 2.0 ** -13 * torch.from_numpy(group_maxima(va.cpu().numpy(), vb.cpu().numpy())).cuda()
        bound = bound + 2.0 ** -8 * (ref.abs() + bound)
    da, db = Device.of(a, sa, 1, ca, spare), Device.of(b, sb, brb, "e4m3", spare)
    c = torch.full((m + 1, n + spare), 7.0, dtype=DTYPES[dtype][1], device="cuda")
    for _ in range(2):
        B.ee_scaled_matmul(da.c, db.c, c, DTYPES[dtype][0], n + spare, 0, stream())
    err = (c[:m, :n].double() - ref).abs()
    assert bool((err <= bound).all()), (float(err.max()), float(bound.min()), int((err > bound).sum()))
    assert bool((c[m] == 7).all()) and bool((c[:, n:] == 7).all())


@pytest.mark.parametrize("m,n,k,ca,spare", [
    (1030, 9000, 1100, "e4m3", 0), (1030, 9001, 1536, "e5m2", 16), (2049, 6104, 1024, "e4m3", 0), (900, 33001, 1040, "e4m3", 32),
    (520, 16800, 1033, "e5m2", 0), (4100, 2300, 1208, "e4m3", 16),
])
def test_bf16_products_of_large_tiles(m, n, k, ca, spare):
    """The 256 x 256 tile: ragged in every direction, even and odd numbers of stages, sums that end inside a stage."""
    say(f"case: scaled matmul big {m}x{n}x{k} {ca} spare {spare}")
    assert tile_of(False, False, n, m, k) == 0
    check_product(m, n, k, ca, 128, "bf16", spare)


# (tile, rows of a, rows of b, depth), for either type of C
TILES = [(2, 262, 13273, 47), (3, 133, 8379, 175), (3, 140, 8379, 513), (4, 834, 1161, 300), (6, 19, 8577, 320), (7, 35, 4207, 200),
         (7, 64, 5001, 2064), (8, 70, 1500, 1500), (8, 200, 1001, 500), (9, 17, 33, 32), (9, 12, 4001, 4100), (10, 3, 40001, 1100),
         (10, 9, 12001, 2048), (11, 1, 32, 32), (11, 14, 20001, 500), (12, 1, 33, 723), (12, 5, 700, 3000)]
TILES_F32 = [(1, 131, 23217, 1675), (1, 1147, 4037, 6348), (5, 241, 4003, 851)]
TILES_BF16 = [(5, 170, 4621, 637), (5, 36, 8359, 80)]


@pytest.mark.parametrize("ca,brb", [("e4m3", 128), ("e5m2", 1)])
@pytest.mark.parametrize("dtype,tile,m,n,k", [("f32", *t) for t in TILES + TILES_F32] + [("bf16", *t) for t in TILES + TILES_BF16])
def test_every_tile(dtype, tile, m, n, k, ca, brb):
    say(f"case: scaled matmul tile {tile} {m}x{n}x{k} {ca} {brb} {dtype}")
    assert tile_of(dtype == "f32", brb == 1, n, m, k) == tile
    check_product(m, n, k, ca, brb, dtype)


@pytest.mark.parametrize("m,n,k", [(3, 130, 300), (70, 333, 1000), (300, 600, 520)])
def test_strides_accumulate_and_columns_past_the_last(m, n, k):
    say(f"case: scaled matmul strides {m}x{n}x{k}")
    a, sa, b, sb = operands(m, n, k, "e4m3", 1, 128, 5)
    ref, bound = reference(a, sa, 1, b, sb, 128)
    da, db = Device.of(a, sa, 1, "e4m3", 32), Device.of(b, sb, 128, "e4m3", 48)
    for ldc in (n + 2, n + 6):       # groups of four features aligned only in the second
        c = torch.full((m, ldc), 3.0, device="cuda")
        B.ee_scaled_matmul(da.c, db.c, c, B.EE_F32, ldc, 0, stream())
        B.ee_scaled_matmul(da.c, db.c, c, B.EE_F32, ldc, 1, stream())
        got = c.double().cpu().numpy()
        assert (np.abs(got[:, :n] - 2 * ref) <= 2 * bound + 2.0 ** -23 * np.abs(ref)).all()
        assert (got[:, n:] == 3).all()


def test_nan_and_infinite_blocks_stay_in_their_rows():
    a, sa, b, sb = operands(40, 200, 300, "e4m3", 1, 128, 9)
    da, db = Device.of(a, sa, 1, "e4m3"), Device.of(b, sb, 128, "e4m3")
    clean = torch.zeros(40, 200, device="cuda")
    B.ee_scaled_matmul(da.c, db.c, clean, B.EE_F32, 200, 0, stream())
    da.data[7, 299] = 0x7F                       # NaN
    da.scale[1, 11] = float("inf")
    c = torch.zeros(40, 200, device="cuda")
    B.ee_scaled_matmul(da.c, db.c, c, B.EE_F32, 200, 0, stream())
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[7, 11]] = True
    assert not torch.isfinite(c[bad]).any() and torch.equal(c[~bad], clean[~bad])


def test_linear_layer_forward_and_both_gradients():
    """Y = X W^T, dX = dY W, dW = dY^T X, all from quantised operands: the formulas,
    and differences of sum(Y dY) along a direction of X and of W."""
    n, i, o = 333, 300, 500
    x, w, dy = matrix(n, i, 1), matrix(o, i, 2, False) * np.float32(0.05), matrix(n, o, 3)
    dev = {k: torch.from_numpy(v).cuda() for k, v in (("x", x), ("w", w), ("dy", dy))}
    xq, xt = Device(n, i, 1, "e4m3"), Device(i, n, 1, "e4m3")
    wq, wt = Device(o, i, 128, "e4m3"), Device(i, o, 128, "e4m3")
    gq, gt = Device(n, o, 1, "e5m2"), Device(o, n, 1, "e5m2")
    B.ee_quantize_blocks(dev["x"], B.EE_F32, n, i, i, xq.c, xt.c, stream())
    B.ee_quantize_blocks(dev["w"], B.EE_F32, o, i, i, wq.c, wt.c, stream())
    B.ee_quantize_blocks(dev["dy"], B.EE_F32, n, o, o, gq.c, gt.c, stream())
    y, dx, dw = (torch.zeros(s, device="cuda") for s in ((n, o), (n, i), (o, i)))
    B.ee_scaled_matmul(xq.c, wq.c, y, B.EE_F32, o, 0, stream())
    B.ee_scaled_matmul(gq.c, wt.c, dx, B.EE_F32, i, 0, stream())
    B.ee_scaled_matmul(gt.c, xt.c, dw, B.EE_F32, i, 0, stream())

    def vals(a, br, code):
        return Q.values(*Q.quantize(np.ascontiguousarray(a), br, code), br)

    for got, a, b, depth in ((y, vals(x, 1, "e4m3"), vals(w, 128, "e4m3"), i), (dx, vals(dy, 1, "e5m2"), vals(w.T, 128, "e4m3"), o),
                             (dw, vals(dy.T, 1, "e5m2"), vals(x.T, 1, "e4m3"), n)):
        ref, mag = Q.matmul(a, b)
        assert (np.abs(got.double().cpu().numpy() - ref) <= (129 + -(-depth // 128)) * 2.0 ** -23 * mag).all()
    # The transposed weight has the weight's own values, so dX is the gradient of
    # sum(Y dY) for the quantised W and dY up to the quantising of dY along the other
    # axis; the difference along a direction is exact, as Y is linear.
    np.testing.assert_array_equal(vals(w, 128, "e4m3"), vals(w.T, 128, "e4m3").T)
    d = matrix(n, i, 4)
    slope = float((d @ vals(w, 128, "e4m3").T * vals(dy, 1, "e5m2")).sum())
    assert abs(float((dx.double().cpu().numpy() * d).sum()) - slope) <= 1e-4 * abs(slope) + 1e-3
    # dW against differences of the unquantised sum(Y dY): each quantised factor is off
    # by at most half a step (2^-4 of e4m3, 2^-3 of e5m2) of each element
    d = matrix(o, i, 5)
    slope = float((x.astype(np.float64) @ d.T * dy).sum())
    terms = float((np.abs(x).astype(np.float64) @ np.abs(d).T * np.abs(dy)).sum())
    assert abs(float((dw.double().cpu().numpy() * d).sum()) - slope) <= (2.0 ** -3 + 2.0 ** -4 + 2.0 ** -7) * terms


def test_captured_product_replays():
    a, sa, b, sb = operands(20, 400, 500, "e4m3", 1, 128, 12)
    da, db = Device.of(a, sa, 1, "e4m3"), Device.of(b, sb, 128, "e4m3")
    x = torch.from_numpy(matrix(20, 500, 13)).cuda()
    c = torch.zeros(20, 400, device="cuda")

    def go():
        B.ee_quantize_blocks(x, B.EE_F32, 20, 500, 500, da.c, None, stream())
        B.ee_scaled_matmul(da.c, db.c, c, B.EE_F32, 400, 0, stream())

    go()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            go()
    for seed in (21, 22, 23):
        x.copy_(torch.from_numpy(matrix(20, 500, seed)))
        c.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = c.clone()
        go()
        torch.cuda.synchronize()
        assert torch.equal(got, c) and got.abs().sum() > 0
