"""ee_exit_logits against the fp64 oracle, and a serving step built of it and
ee_sample.

With the exit's own weights a logit may be off as the decode decision's
(tests/test_gpu_decode.py): c sum_k |W| |z| with c = 2^-8 for a bf16 Norm exit, 2^-6 for
a bf16 MLP exit and 2^-20 else, plus half a step (2^-8 of it) if stored as bf16.

With 8-bit weights the rows are quantised from fp32 values that are off by at most
2^-18 of themselves (norm: sums of 8192 squares at worst) from the oracle's, so a code can
differ by one step only where the oracle's value lies that near a border between two
codes; the scale is off by the same 2^-18; the product as in tests/test_gpu_scaled.py.
"""

import numpy as np
import pytest
import torch

import oracle as O
from oracle import sampling as S
from oracle import scaled as Q
import workloads as W
from paper_2402_00518_amd import binding as B
from paper_2402_00518_amd.session import to_device
from test_gpu_scaled import group_maxima

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)


def make(kind, n, h, V, I, dtype, norm="rms", bias=False, seed=0):
    w = W.custom(kind, n, h, V, I, dtype, (1.0,), row_scale=True, zipf=True, name="logits", norm=norm, bias=bias)
    return W.make_batch(w, seed, random_gamma=True)


def device_exit(b, own_w=True):
    w, p = b.workload, b.exits[0]
    d = {"w_out": p.w_out if own_w else None, "gamma": p.gamma, "gamma_mlp": p.gamma_mlp, "w_gate": p.w_gate, "w_up": p.w_up,
         "w_down": p.w_down, "beta": p.beta}
    t = {k: to_device(a, "cuda") for k, a in d.items() if a is not None}
    dtype = B.EE_F32 if w.dtype == "f32" else B.EE_BF16
    norm = B.EE_NORM_LAYER if w.norm == "layer" else B.EE_NORM_RMS
    return B.make_exit(w.kind, dtype, w.hidden, w.vocab, w.intermediate if w.kind == B.EE_EXIT_MLP else 0, w.eps, norm=norm, **t), t


def logits(e, w_out, x, n, V, dtype, ld):
    nb = B.ee_logits_workspace_bytes(e, w_out, n)
    ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full((n + 1, ld), 5.0, dtype=torch.float32 if dtype == B.EE_F32 else torch.bfloat16, device="cuda")
    B.ee_exit_logits(e, w_out, x, n, out, dtype, ld, ws, nb, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (out[n] == 5).all() and (out[:n, V:] == 5).all()
    return out[:n, :V]


CASES = [
    ("norm_one_row", W.EXIT_NORM, 1, 64, 50, 0, "bf16"),
    ("norm_ragged", W.EXIT_NORM, 5, 192, 1003, 0, "bf16"),
    ("norm_70_rows", W.EXIT_NORM, 70, 128, 5001, 0, "bf16"),
    ("norm_200_rows", W.EXIT_NORM, 200, 1024, 9000, 0, "bf16"),
    ("norm_vocab_one", W.EXIT_NORM, 3, 64, 1, 0, "bf16"),
    ("norm_wide_vocab", W.EXIT_NORM, 20, 128, 40002, 0, "bf16"),
    ("norm_max_hidden", W.EXIT_NORM, 3, 32768, 300, 0, "bf16"),
    ("embedding", W.EXIT_EMBEDDING, 9, 320, 500, 0, "bf16"),
    ("layernorm_bias", W.EXIT_NORM, 9, 192, 1000, 0, "bf16"),
    ("norm_f32", W.EXIT_NORM, 6, 64, 333, 0, "f32"),
    ("embedding_f32", W.EXIT_EMBEDDING, 2, 64, 129, 0, "f32"),
    ("layernorm_bias_f32", W.EXIT_NORM, 40, 2112, 333, 0, "f32"),
    ("mlp", W.EXIT_MLP, 7, 192, 900, 320, "bf16"),
    ("mlp_split", W.EXIT_MLP, 50, 1024, 700, 4096, "bf16"),
    ("mlp_f32", W.EXIT_MLP, 33, 128, 300, 192, "f32"),
]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("name,kind,n,h,V,I,dtype", CASES, ids=[c[0] for c in CASES])
def test_own_weights(name, kind, n, h, V, I, dtype, out):
    say(f"case: exit logits {name} {out}")
    bias = "layernorm" in name
    b = make(kind, n, h, V, I, dtype, "layer" if bias else "rms", bias)
    e, keep = device_exit(b)
    got = logits(e, None, to_device(b.hidden[0], "cuda"), n, V, B.EE_F32 if out == "f32" else B.EE_BF16, V + (1 if n % 2 else 4))
    ex = O.exits_from_batch(b)[0]
    f = O.exit_forward(ex, W.decode(b.hidden[0]))
    c = 2.0 ** -20 if dtype == "f32" or kind == W.EXIT_EMBEDDING else 2.0 ** -6 if kind == W.EXIT_MLP else 2.0 ** -8
    bound = c * (np.abs(f["z"]) @ np.abs(ex.w_out).T)
    if out == "bf16":
        bound = bound + 2.0 ** -8 * (np.abs(f["s"]) + bound)
    err = np.abs(got.double().cpu().numpy() - f["s"])
    assert (err <= bound).all(), (err.max(), bound.max())


def scaled_w(b):
    w = W.decode(b.exits[0].w_out).astype(np.float32)
    codes, scale = Q.quantize(w, 128, "e4m3")
    t = torch.from_numpy(Q.encode(codes, "e4m3")).cuda(), torch.from_numpy(scale).cuda()
    return B.make_scaled(*t, block_rows=128), t, Q.values(codes, scale, 128)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("name,kind,n,h,V,I,dtype", [c for c in CASES if c[1] != W.EXIT_MLP or c[6] == "f32"],
                         ids=[c[0] for c in CASES if c[1] != W.EXIT_MLP or c[6] == "f32"])
def test_8_bit_weights(name, kind, n, h, V, I, dtype, out):
    say(f"case: exit logits 8-bit {name} {out}")
    bias = "layernorm" in name
    b = make(kind, n, h, V, I, dtype, "layer" if bias else "rms", bias, seed=1)
    e, keep = device_exit(b, own_w=False)
    wq, tensors, wv = scaled_w(b)
    got = logits(e, wq, to_device(b.hidden[0], "cuda"), n, V, B.EE_F32 if out == "f32" else B.EE_BF16, V + (3 if n % 2 else 0))
    z = O.exit_forward(O.exits_from_batch(b)[0], W.decode(b.hidden[0]))["z"]
    codes, scale = Q.quantize(z.astype(np.float32), 1, "e4m3")
    y = z * Q.expand(1.0 / scale.astype(np.float64), n, h, 1)
    step = Q.step_of(y, "e4m3")
    off = np.abs(np.abs(y - codes) - step / 2)                # distance from the nearest border inside the step
    flip = off <= 2.0 ** -17 * np.abs(y) + 1e-12
    s = Q.expand(scale.astype(np.float64), n, h, 1)
    dz = np.where(flip, step * s * 2, 0.0) + 2.0 ** -18 * np.abs(codes * s)
    ref = (codes * s) @ wv.T
    mag = np.abs(codes * s) @ np.abs(wv).T
    bound = dz @ np.abs(wv).T + (129 + scale.shape[0]) * 2.0 ** -23 * mag
    if out == "bf16":
        bound = bound + 7 * 2.0 ** -13 * group_maxima(codes * s, wv)
        bound = bound + 2.0 ** -8 * (np.abs(ref) + bound)
    err = np.abs(got.double().cpu().numpy() - ref)
    assert (err <= bound).all(), (err.max(), bound.max(), flip.mean())


@pytest.mark.parametrize("n", [1, 37])
def test_8_bit_weights_behind_a_bf16_mlp(n):
    """The rows of a bf16 MLP exit carry its own roundings (2^-6 of them at most, twice the
    exit's), each of which may move a code by as much as half a step more on either side."""
    h, V, I = 256, 900, 512
    b = make(W.EXIT_MLP, n, h, V, I, "bf16", seed=2)
    e, keep = device_exit(b, own_w=False)
    wq, tensors, wv = scaled_w(b)
    got = logits(e, wq, to_device(b.hidden[0], "cuda"), n, V, B.EE_F32, V).double().cpu().numpy()
    z = O.exit_forward(O.exits_from_batch(b)[0], W.decode(b.hidden[0]))["z"]
    top = np.abs(z).reshape(n, -1, 128).max(2).repeat(128, 1)
    dz = 2.0 ** -6 * np.abs(z).max(1, keepdims=True) + 2.0 ** -4 * np.abs(z) + 2.0 ** -10 * top / 448
    assert (np.abs(got - z @ wv.T) <= dz @ np.abs(wv).T).all()
    assert np.linalg.norm(got - z @ wv.T) <= 0.05 * np.linalg.norm(z @ wv.T)


@pytest.mark.parametrize("scaled", [False, True])
def test_serving_step(scaled):
    """Hidden states -> logits -> token, confidence and exit flag, as a server calls them, eagerly and captured; a greedy
    request answers what the decode decision answers."""
    n, h, V = 24, 256, 3000
    b = make(W.EXIT_NORM, n, h, V, 0, "bf16", seed=3)
    e, keep = device_exit(b, own_w=not scaled)
    wq, tensors, wv = scaled_w(b)
    x = to_device(b.hidden[0], "cuda")
    w = wq if scaled else None
    nb = max(B.ee_logits_workspace_bytes(e, w, n), B.ee_sample_workspace_bytes(n, V))
    ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.zeros(n, V, device="cuda")
    g = np.random.default_rng(0)
    temperature = torch.tensor(g.choice([0.0, 0.7, 1.0], n), dtype=torch.float32, device="cuda")
    top_k, top_p = torch.full((n,), 40, dtype=torch.int32, device="cuda"), torch.full((n,), 0.95, device="cuda")
    how = B.make_sampling(temperature, top_k, top_p)
    u = torch.tensor(g.random(n), dtype=torch.float32, device="cuda")
    token, flag = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))
    prob, conf = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")

    def step():
        s = torch.cuda.current_stream().cuda_stream
        B.ee_exit_logits(e, w, x, n, out, B.EE_F32, V, ws, nb, s)
        B.ee_sample(out, B.EE_F32, n, V, V, None, 0, how, u, 0.02, token, prob, conf, flag, ws, nb, s)

    step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for _ in range(3):
        u.uniform_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (out, token, prob, conf, flag)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (out, token, prob, conf, flag)))
        host = out.double().cpu().numpy()
        for r in range(n):
            want = S.sample(host[r], float(u[r]), temperature=float(temperature[r]), top_k=40, top_p=float(top_p[r]))
            assert want[3] < 1e-9 or int(token[r]) == want[0]
            assert abs(float(conf[r]) - want[2]) <= 2.0 ** -22 * want[2]
            assert int(flag[r]) == (float(conf[r]) > np.float32(0.02))
    if not scaled:
        wb = B.ee_decode_workspace_bytes(e, n)
        dws = torch.empty(wb, dtype=torch.uint8, device="cuda")
        t2, c2, f2 = torch.zeros_like(token), torch.zeros_like(conf), torch.zeros_like(flag)
        B.ee_exit_decide(e, x, n, 0.02, t2, c2, f2, dws, wb, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        greedy = (temperature <= 0).cpu().numpy()
        top2 = np.sort(host, axis=1)[:, -2:]
        clear = greedy & (top2[:, 1] - top2[:, 0] > 1e-4)      # both are fp32 sums of the same terms
        assert clear.any() and (t2.cpu().numpy()[clear] == token.cpu().numpy()[clear]).all()
        # fp32 sums of 256 terms and exponentials: well inside 1e-5
        assert torch.allclose(conf, c2, rtol=1e-5, atol=0)
