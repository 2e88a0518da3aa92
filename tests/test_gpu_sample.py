"""ee_sample against the fp64 oracle: the token must be the oracle's (cases lie
further than 1e-9 of the kept mass from a border, or are left out and counted),
the probability and the confidence equal to a rounding to fp32 (2^-24) and the 1e-12
that the masses' exponentials are off by: 2^-22 relative."""

import numpy as np
import pytest
import torch

from oracle import sampling as S
from paper_2402_00518_amd import binding as B

pytestmark = pytest.mark.gpu

DTYPES = {"f32": (B.EE_F32, torch.float32), "bf16": (B.EE_BF16, torch.bfloat16)}
TOL = 2.0 ** -22


def say(msg):
    print(msg, flush=True)


def dev(a, dtype):
    return None if a is None else torch.as_tensor(np.asarray(a), dtype=dtype, device="cuda")


def pack(allowed):
    n, v = allowed.shape
    bits = np.zeros((n, -(-v // 32) * 32), dtype=np.uint8)
    bits[:, :v] = allowed
    bits[:, v:] = 1                       # bits past the vocabulary do not matter
    return np.packbits(bits, axis=1, bitorder="little").view(np.int32)


def run(x, u, allowed=None, temperature=None, top_k=None, top_p=None, min_p=None, threshold=0.3, ld=None, ws=None):
    """x: device logits [n][ld]; the rest host arrays of n or None."""
    n = x.shape[0]
    v = x.shape[1] if ld is None else ld[0]
    words = None if allowed is None else torch.from_numpy(pack(allowed)).cuda()
    par = [dev(temperature, torch.float32), dev(top_k, torch.int32), dev(top_p, torch.float32), dev(min_p, torch.float32)]
    how = B.make_sampling(*par)
    out = [torch.full((n,), 9, dtype=torch.int32, device="cuda"), torch.full((n,), 9.0, device="cuda"),
           torch.full((n,), 9.0, device="cuda"), torch.full((n,), 9, dtype=torch.int32, device="cuda")]
    ud = dev(u, torch.float32)
    nb = B.ee_sample_workspace_bytes(n, v)
    ws = torch.full((nb,), 0xA5, dtype=torch.uint8, device="cuda") if ws is None else ws
    dtype = B.EE_F32 if x.dtype == torch.float32 else B.EE_BF16
    B.ee_sample(x, dtype, n, v, x.shape[1], words, 0 if words is None else words.shape[1], how, ud, threshold, *out, ws,
                ws.numel(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return [o.cpu().numpy() for o in out]


def check(x, u, got, allowed=None, threshold=0.3, vocab=None, **how):
    host = x.float().cpu().numpy().astype(np.float64)[:, :vocab]
    left_out = 0
    for r in range(host.shape[0]):
        par = {k: float(np.float32(v[r])) if k != "top_k" else int(v[r]) for k, v in how.items() if v is not None}
        token, prob, conf, gap = S.sample(host[r], float(np.float32(u[r])), None if allowed is None else allowed[r], **par)
        at = (r, par, float(u[r]))
        if gap < 1e-9:
            left_out += 1
        else:
            assert got[0][r] == token, (at, got[0][r], token, gap)
            assert abs(got[1][r] - prob) <= TOL * prob, (at, got[1][r], prob)
        assert abs(got[2][r] - conf) <= TOL * conf, (at, got[2][r], conf)
        assert got[3][r] == (got[2][r] > np.float32(threshold)), at
    assert left_out <= 1 + host.shape[0] // 50


def params(n, g, kind):
    how = {"temperature": None, "top_k": None, "top_p": None, "min_p": None}
    if kind in ("mixed", "temperature"):
        how["temperature"] = g.choice([0.0, 0.3, 0.7, 1.0, 1.0, 1.5, 8.0], n).astype(np.float32)
    if kind in ("mixed", "top_k"):
        how["top_k"] = g.choice([0, 1, 2, 5, 40, 64, 1000], n).astype(np.int32)
    if kind in ("mixed", "top_p"):
        how["top_p"] = g.choice([1.0, 0.95, 0.9, 0.5, 0.05, 0.0], n).astype(np.float32)
    if kind in ("mixed", "min_p"):
        how["min_p"] = g.choice([0.0, 0.01, 0.2, 1.0, 2.0], n).astype(np.float32)
    return how


def logits(n, v, g, sigma=2.5, peaks=8):
    x = g.standard_normal((n, v)) * sigma
    for r in range(n):
        x[r, g.integers(0, v, min(peaks, v))] += g.uniform(2, 10, min(peaks, v))
    return x.astype(np.float32)


@pytest.mark.parametrize("kind", ["none", "temperature", "top_k", "top_p", "min_p", "mixed"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", [(3, 1), (5, 2), (4, 63), (4, 65), (7, 255), (6, 1000), (40, 4097), (12, 32000), (5, 50021)])
def test_sizes_and_filters(n, v, dtype, kind):
    say(f"case: sample {n}x{v} {dtype} {kind}")
    g = np.random.default_rng(n * 1000 + v)
    x = torch.from_numpy(logits(n, v, g)).cuda().to(DTYPES[dtype][1])
    u = g.random(n).astype(np.float32)
    how = params(n, g, kind)
    check(x, u, run(x, u, **how), **how)


@pytest.mark.parametrize("n,v,sigma,kind", [
    (2, 131072, 3.0, "top_p"), (3, 200000, 0.4, "top_p"), (2, 1 << 20, 2.0, "mixed"), (2, 1 << 20, 1.0, "none"),
    (4, 40000, 1e-3, "top_p"), (3, 70000, 0.0, "top_p"), (3, 70000, 0.0, "none"), (6, 33333, 0.02, "mixed"),
])
def test_flat_and_long_rows(n, v, sigma, kind):
    """Nuclei of tens of thousands of tokens, thousands of equal logits, a million ids."""
    say(f"case: sample flat {n}x{v} sigma {sigma} {kind}")
    g = np.random.default_rng(v)
    x = torch.from_numpy(logits(n, v, g, sigma, 0)).cuda()
    u = g.random(n).astype(np.float32)
    how = params(n, g, kind)
    check(x, u, run(x, u, **how), **how)
    h = x.bfloat16()
    check(h, u, run(h, u, **how), **how)


@pytest.mark.parametrize("top_k,top_p", [(4095, 1.0), (4096, 1.0), (4097, 1.0), (20000, 1.0), (20000, 0.9), (20000, 0.01), (30000, 0.999),
                                         (29999, 0.5), (40000, 0.9)])
@pytest.mark.parametrize("sigma", [2.0, 1e-4, 0.0])
def test_thousands_of_kept_tokens(top_k, top_p, sigma):
    say(f"case: sample top_k {top_k} top_p {top_p} sigma {sigma}")
    n, v = 4, 30000
    g = np.random.default_rng(top_k)
    x = torch.from_numpy(logits(n, v, g, sigma, 0)).cuda()
    if sigma == 1e-4:
        x[:, ::3] = x[:, :1]            # a third of the row is equal
    u = g.random(n).astype(np.float32)
    how = {"top_k": np.full(n, top_k), "top_p": np.full(n, top_p)}
    check(x, u, run(x, u, **how), **how)


def test_cut_far_below_the_maximum():
    """A sharp temperature: what top-k keeps lies thousands of units below the largest."""
    n, v = 6, 20000
    g = np.random.default_rng(3)
    x = torch.from_numpy(logits(n, v, g, 2.0, 3)).cuda()
    u = g.random(n).astype(np.float32)
    for t in (0.01, 1e-3, 1e-30, 1e-44):
        for k in (3, 500, 10000):
            how = {"temperature": np.full(n, t), "top_k": np.full(n, k), "top_p": np.array([1.0, 0.9, 0.999999, 0.5, 1.0, 0.99])}
            check(x, u, run(x, u, **how), **how)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks(dtype):
    n, v = 12, 3001
    g = np.random.default_rng(8)
    x = logits(n, v, g)
    allowed = g.random((n, v)) < 0.5
    allowed[1] = False                        # nothing left
    allowed[2] = False
    allowed[2, 3000] = True                   # one token
    x[3, ~allowed[3]] = np.nan                # what is not allowed does not matter
    x[4, ~allowed[4]] = np.inf
    x[5, g.random(v) < 0.9] = -np.inf         # banned by their logits
    x[6] = -np.inf                            # all of them
    x[7, g.random(v) < 0.9] = np.finfo(np.float32).min if dtype == "f32" else -3.3895e38
    x[8] = np.finfo(np.float32).min if dtype == "f32" else -3.3895e38
    x[9, np.flatnonzero(allowed[9])[5]] = np.nan
    x[10, np.flatnonzero(allowed[10])[5]] = np.inf
    d = torch.from_numpy(x).cuda().to(DTYPES[dtype][1])
    u = g.random(n).astype(np.float32)
    for kind in ("none", "top_k", "top_p", "mixed"):
        how = params(n, g, kind)
        got = run(d, u, allowed, **how)
        check(d, u, got, allowed, **how)
        for r in (1, 6, 9, 10):
            assert got[0][r] == -1 and got[1][r] == 0 and got[2][r] == 0 and got[3][r] == 0
        assert got[0][2] == 3000


def test_parameters_out_of_range():
    n, v = 14, 500
    g = np.random.default_rng(4)
    x = torch.from_numpy(logits(n, v, g)).cuda()
    u = g.random(n).astype(np.float32)
    u[9], u[10], u[11], u[12] = 1.0, 5.0, -3.0, np.nan
    how = {"temperature": np.array([np.inf, -1, 1, 1, 1, 1, 1, 1, np.nan, 1, 1, 1, 1, 1]),
           "top_k": np.array([0, 3, -5, 1 << 30, 3, 3, 3, 0, 0, 0, 0, 5, 0, 0]),
           "top_p": np.array([1, 1, 1, 1, -1, 7, np.nan, 0.9, 1, 1, 1, 1, 1, 1]),
           "min_p": np.array([0, 0, 0, 0, 0, 0, 0, np.nan, 0, 0, 0, 0, 0, -1])}
    got = run(x, u, **how)
    for r in (6, 7, 8, 12):
        assert got[0][r] == -1 and got[1][r] == 0 and got[2][r] == 0
    rest = [r for r in range(n) if r not in (6, 7, 8, 12)]
    check(x[rest], np.clip(u[rest], 0, None), [o[rest] for o in got], **{k: a[rest] for k, a in how.items()})


def test_ties_and_signed_zeros():
    x = torch.tensor([[0.0, -0.0, 1.0, 1.0, 1.0, -0.0]] * 6, device="cuda")
    u = np.array([0.0, 0.3, 0.34, 0.6, 0.7, 0.999], dtype=np.float32)
    how = {"top_k": np.array([2, 3, 4, 4, 5, 5])}
    check(x, u, run(x, u, **how), **how)
    got = run(x, np.full(6, 0.9999, np.float32), top_k=np.array([1, 2, 3, 4, 5, 6]))
    assert got[0].tolist() == [2, 3, 4, 4, 4, 5]          # after the ones come ids 0, 1, 5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_rows_of_nan_past_the_vocabulary(dtype):
    g = np.random.default_rng(6)
    for v, ld in ((1000, 1001), (1000, 1004), (999, 1000), (33, 35)):
        full = np.full((5, ld), np.nan, dtype=np.float32)
        full[:, :v] = logits(5, v, g)
        x = torch.from_numpy(full).cuda().to(DTYPES[dtype][1])
        u = g.random(5).astype(np.float32)
        how = params(5, g, "mixed")
        check(x, u, run(x, u, ld=(v,), **how), vocab=v, **how)


def test_frequencies_follow_the_kept_distribution():
    """4096 evenly spaced numbers hit every kept token as often as its share says, to within one."""
    x = torch.randn(1, 200, generator=torch.Generator().manual_seed(1)).mul(2).cuda()
    n = 4096
    rows = x.expand(n, -1).contiguous()
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    got = run(rows, u, top_k=np.full(n, 50), top_p=np.full(n, 0.9))[0]
    mass = S.kept_mass(x[0].double().cpu().numpy(), top_k=50, top_p=float(np.float32(0.9)))
    share = np.bincount(got, minlength=200)
    assert (np.abs(share - mass / mass.sum() * n) <= 1).all()


def test_equal_calls_and_replays_give_equal_results():
    g = np.random.default_rng(2)
    n, v = 9, 60000
    x = torch.from_numpy(logits(n, v, g, 0.5)).cuda()
    u = dev(g.random(n), torch.float32)
    top_p = dev(np.full(n, 0.9), torch.float32)
    how = B.make_sampling(top_p=top_p)
    nb = B.ee_sample_workspace_bytes(n, v)
    ws = torch.zeros(nb, dtype=torch.uint8, device="cuda")
    token, prob = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")

    def go():
        B.ee_sample(x, B.EE_F32, n, v, v, None, 0, how, u, 0.5, token, prob, None, None, ws, nb,
                    torch.cuda.current_stream().cuda_stream)

    go()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            go()
    for k in range(3):
        x.copy_(torch.from_numpy(logits(n, v, g, 0.5 + k)))
        u.uniform_()
        token.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        a = token.clone(), prob.clone()
        go()
        torch.cuda.synchronize()
        assert torch.equal(a[0], token) and torch.equal(a[1], prob) and (token >= 0).all()


@pytest.mark.parametrize("n,v,ld", [(1, 64001, 64001), (4, 256001, 256004), (64, 40961, 40962), (65, 40961, 40964)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["none", "top_p", "mixed"])
def test_rows_that_several_blocks_read(n, v, ld, dtype, kind):
    """Long rows, few of them: random numbers at both ends, a mask, and rows with no
    distribution, by what lies in the first ids, in the middle and in the last ones."""
    say(f"case: sample long {n}x{v} ld {ld} {dtype} {kind}")
    g = np.random.default_rng(n + v)
    x = torch.full((n, ld), float("nan"), device="cuda")
    x[:, :v] = torch.from_numpy(logits(n, v, g)).cuda()
    x = x.to(DTYPES[dtype][1])
    u = g.random(n).astype(np.float32)
    u[0] = np.nextafter(np.float32(1.0), np.float32(0.0))
    u[n // 2] = 0.0
    allowed = g.random((n, v)) < 0.7
    allowed[:, v // 3] = True
    how = params(n, g, kind)
    check(x, u, run(x, u, ld=(v,), **how), vocab=v, **how)
    check(x, u, run(x, u, allowed, ld=(v,), **how), allowed, vocab=v, **how)
    if n < 3:
        return
    bad = x.clone()
    bad[0, v - 1] = float("nan")
    bad[1, 0] = float("inf")
    bad[2, :v] = float("-inf")
    allowed[3] = False
    got = run(bad, u, allowed | (np.arange(n) < 3)[:, None], ld=(v,), **how)
    for r in range(4):
        assert [float(o[r]) for o in got] == [-1, 0, 0, 0], r
    rest = {k: None if a is None else a[4:] for k, a in how.items()}
    check(bad[4:], u[4:], [o[4:] for o in got], allowed[4:], vocab=v, **rest)
