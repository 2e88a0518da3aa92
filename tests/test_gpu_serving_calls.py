"""Calls of the 8-bit products, the exit logits and the sampling that one call at a time on
compact matrices does not make: rows that lie 2^31 elements apart, two streams at
once, two captured graphs that share a workspace.  Each is compared, bit for bit, with the
same call made the plain way, which the other tests hold against the oracle.
"""

import numpy as np
import pytest
import torch

from paper_2402_00518_amd import binding as B

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)


def stream():
    return torch.cuda.current_stream().cuda_stream


def far(rows, cols, dtype, seed=None):
    """[rows][cols] within rows that lie so far apart that the last starts past element 2^31."""
    ld = (2 ** 31 // (rows - 1) + 16) // 8 * 8 + 8
    x = torch.empty((rows - 1) * ld + cols, dtype=dtype, device="cuda").as_strided((rows, cols), (ld, 1))
    assert (rows - 1) * ld >= 2 ** 31
    if seed is not None:
        x.copy_(torch.from_numpy(np.random.default_rng(seed).standard_normal((rows, cols)).astype(np.float32)).cuda())
    return x, ld


class Matrix:
    """8-bit codes of x, quantised on the device."""

    def __init__(self, x, block_rows):
        rows, cols = x.shape
        ld = -(-cols // 16) * 16
        self.q = torch.zeros(rows, ld, dtype=torch.uint8, device="cuda")
        self.scale = torch.zeros(-(-cols // 128), -(-rows // block_rows), device="cuda")
        self.c = B.make_scaled(self.q[:, :cols], self.scale, block_rows, B.EE_E4M3)
        if x.stride(0) == cols:
            B.ee_quantize_blocks(x, B.EE_F32, rows, cols, cols, self.c, None, stream())


def normal(rows, cols, seed):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal((rows, cols)).astype(np.float32)).cuda()


def sampler(x, ld, v, seed):
    """(call, outputs) of one sampling of x's rows."""
    n = x.shape[0]
    g = np.random.default_rng(seed)
    u = torch.from_numpy(g.random(n).astype(np.float32)).cuda()
    top_p = torch.full((n,), 0.9, device="cuda")
    how = B.make_sampling(top_p=top_p)
    out = [torch.zeros(n, dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.float32, torch.int32)]
    dtype = B.EE_F32 if x.dtype == torch.float32 else B.EE_BF16
    nb = B.ee_sample_workspace_bytes(n, v)

    def call(ws=None, keep=[u, top_p]):
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda") if ws is None else ws
        B.ee_sample(x, dtype, n, v, ld, None, 0, how, u, 0.1, *out, ws, ws.numel(), stream())
        return ws

    return call, out


@pytest.mark.parametrize("n,v", [(9, 1000), (9, 70001)])
def test_sampling_of_rows_far_apart(n, v):
    say(f"case: sample rows far apart {n}x{v}")
    x, ld = far(n, v, torch.bfloat16, seed=1)
    near = x.contiguous()
    a, got = sampler(x, ld, v, 2)
    b, want = sampler(near, v, v, 2)
    keep = a(), b()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and (got[0] >= 0).all() and len(keep) == 2


@pytest.mark.parametrize("n", [9, 40, 200])
@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
def test_logits_of_rows_far_apart(n, out_dtype):
    say(f"case: logits rows far apart {n} {out_dtype}")
    h, v = 128, 1000
    dtype = B.EE_F32 if out_dtype == "f32" else B.EE_BF16
    w, x = normal(v, h, 3).bfloat16(), normal(n, h, 4).bfloat16()
    e = B.make_exit(B.EE_EXIT_EMBEDDING, B.EE_BF16, h, v, 0, 1e-5, w_out=w)
    wq = Matrix(w.float(), 128)
    got, ld = far(n, v, torch.float32 if out_dtype == "f32" else torch.bfloat16)
    want = torch.zeros(n, v, dtype=got.dtype, device="cuda")
    for m in (None, wq.c):
        nb = B.ee_logits_workspace_bytes(e, m, n)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
        B.ee_exit_logits(e, m, x, n, got, dtype, ld, ws, nb, stream())
        B.ee_exit_logits(e, m, x, n, want, dtype, v, ws, nb, stream())
        torch.cuda.synchronize()
        assert torch.equal(got, want) and want.float().abs().sum() > 0


@pytest.mark.parametrize("m,n", [(9, 1000), (40, 300), (300, 520)])
@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
def test_product_with_rows_far_apart(m, n, out_dtype):
    say(f"case: product rows far apart {m}x{n} {out_dtype}")
    k = 1040
    dtype = B.EE_F32 if out_dtype == "f32" else B.EE_BF16
    a, b = Matrix(normal(m, k, 5), 1), Matrix(normal(n, k, 6), 128)
    got, ld = far(m, n, torch.float32 if out_dtype == "f32" else torch.bfloat16)
    want = torch.zeros(m, n, dtype=got.dtype, device="cuda")
    B.ee_scaled_matmul(a.c, b.c, got, dtype, ld, 0, stream())
    B.ee_scaled_matmul(a.c, b.c, want, dtype, n, 0, stream())
    torch.cuda.synchronize()
    assert torch.equal(got, want) and want.float().abs().sum() > 0


@pytest.mark.parametrize("rows,cols", [(9, 200), (130, 130)])
def test_codes_of_rows_far_apart(rows, cols):
    say(f"case: codes of rows far apart {rows}x{cols}")
    x, ld = far(rows, cols, torch.float32, seed=7)
    near = Matrix(x.contiguous(), 1)
    got, turned = Matrix(x, 1), Matrix(x.t(), 1)
    want_turned = Matrix(x.t().contiguous(), 1)
    B.ee_quantize_blocks(x, B.EE_F32, rows, cols, ld, got.c, turned.c, stream())
    torch.cuda.synchronize()
    assert torch.equal(got.q, near.q) and torch.equal(got.scale, near.scale) and near.q.any()
    assert torch.equal(turned.q, want_turned.q) and torch.equal(turned.scale, want_turned.scale)


def test_two_streams_at_once():
    """Products, logits and samplings of different inputs on two streams, none waiting for the other."""
    say("case: two streams")
    h, v, n = 512, 45000, 20
    sides = []
    for seed in (10, 20):
        w, x = normal(v, h, seed), normal(n, h, seed + 1).bfloat16()
        wq = Matrix(w, 128)
        gamma = torch.ones(h, device="cuda").bfloat16()
        e = B.make_exit(B.EE_EXIT_NORM, B.EE_BF16, h, v, 0, 1e-5, gamma=gamma)
        out = torch.zeros(n, v, device="cuda")
        nb = B.ee_logits_workspace_bytes(e, wq.c, n)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
        draw, got = sampler(out, v, v, seed + 2)
        sws = torch.empty(B.ee_sample_workspace_bytes(n, v), dtype=torch.uint8, device="cuda")
        big = Matrix(normal(700, h, seed + 3), 1)
        c = torch.zeros(700, v, device="cuda")
        sides.append((e, wq, x, out, nb, ws, draw, got, sws, big, c, gamma))

    def go(s):
        e, wq, x, out, nb, ws, draw, got, sws, big, c, _ = s
        B.ee_scaled_matmul(big.c, wq.c, c, B.EE_F32, v, 0, stream())
        B.ee_exit_logits(e, wq.c, x, n, out, B.EE_F32, v, ws, nb, stream())
        draw(sws)

    want = []
    for s in sides:
        go(s)
        torch.cuda.synchronize()
        want.append([t.clone() for t in (s[3], *s[7], s[10])])
    streams = [torch.cuda.Stream() for _ in sides]
    for _ in range(3):
        for s in sides:
            for t in (s[3], *s[7], s[10]):
                t.zero_()
        torch.cuda.synchronize()
        for _ in range(4):
            for side, s in zip(streams, sides):
                with torch.cuda.stream(side):
                    go(s)
        torch.cuda.synchronize()
        for s, w in zip(sides, want):
            assert all(torch.equal(a, b) for a, b in zip((s[3], *s[7], s[10]), w))
    assert not torch.equal(want[0][0], want[1][0])


def test_two_graphs_that_share_a_workspace():
    """Long rows (whose maxima, sums and counts pass through the workspace) sampled by two captured graphs, in turn with
    eager calls, all on one stream with one workspace."""
    say("case: two graphs, one workspace")
    shapes = ((3, 90000), (20, 50021))
    calls = [sampler(normal(n, v, n) * 3, v, v, n + 1) for n, v in shapes]
    ws = torch.full((max(B.ee_sample_workspace_bytes(*s) for s in shapes),), 0xA5, dtype=torch.uint8, device="cuda")
    want = []
    for call, out in calls:
        call(ws)
        torch.cuda.synchronize()
        want.append([t.clone() for t in out])
    side = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(side):
        for call, _ in calls:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                call(ws)
            graphs.append(g)
        for k in range(6):
            i = k % 2
            for _, out in calls:
                for t in out:
                    t.zero_()
            graphs[i].replay()
            if k % 3 == 0:
                calls[1 - i][0](ws)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(calls[i][1], want[i]))
            if k % 3 == 0:
                assert all(torch.equal(a, b) for a, b in zip(calls[1 - i][1], want[1 - i]))
