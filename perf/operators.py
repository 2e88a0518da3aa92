"""Performance cases of the operators an exit answers with: 8-bit block-scaled
matrices and sampling.

  quantize  ee_quantize_blocks: a matrix as 8-bit codes with an fp32 scale for
            each block of 128 columns and 1 or 128 rows, as it is, transposed
            or both.
  matmul    ee_scaled_matmul: C = A B^T of two such matrices.
  logits    ee_exit_logits: the logits of an exit, with its output matrix in
            its own type or in 8 bits.
  sample    ee_sample: a token for each row of logits from a given random
            number, by temperature, top-k, top-p and min-p, with the confidence
            and the exit flag of the greedy decision.

Shapes are the exits of this repository's workloads (7B, 13B and 70B sized, a
vocabulary of 32000) and generic ones between and around them.
"""

import math

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-5
BLOCK = 128
TYPES = {"f32": (0, torch.float32, 4), "bf16": (1, torch.bfloat16, 2)}
CODES = {"e4m3": (2, torch.float8_e4m3fn, 448.0), "e5m2": (3, torch.float8_e5m2, 57344.0)}
LEAST = 2.0 ** -100  # the least scale of a block


def _quantize_case(name, rows, cols, dtype, block_rows, code="e4m3", out="as_is"):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "block_rows": block_rows, "code": code, "out": out}


def _matmul_case(name, rows, features, depth, dtype="bf16", code="e4m3", block_rows=128):
    return {"name": name, "op": "matmul", "rows": rows, "features": features, "depth": depth, "dtype": dtype, "code": code,
            "block_rows": block_rows}


def _logits_case(name, kind, rows, hidden, vocab, scaled, dtype="bf16"):
    return {"name": name, "op": "logits", "kind": kind, "rows": rows, "hidden": hidden, "vocab": vocab, "scaled": scaled, "dtype": dtype}


def _sample_case(name, rows, vocab, dtype="f32", filters="mixed", mask=False):
    return {"name": name, "op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "filters": filters, "mask": mask}


def listed():
    return [
        # the rows of a small decoding batch on their way into an 8-bit product: latency
        _quantize_case("quantize_8row", 8, 4096, "bf16", 1),
        # an output matrix laid out once from its fp32 masters
        _quantize_case("quantize_weight_f32", 32000, 4096, "f32", 128),
        # activations of a ragged micro-batch for both products of a training step that read them
        _quantize_case("quantize_both_ragged", 4001, 5120, "bf16", 1, out="both"),
        # one sequence being decoded, the 7B output matrix
        _matmul_case("matmul_1row_7b", 1, 32000, 4096),
        # a serving batch through a down projection: few features, a long sum
        _matmul_case("matmul_48row_down", 48, 5120, 13824, dtype="f32"),
        # the forward product of a training step
        _matmul_case("matmul_4096row_7b", 4096, 32000, 4096),
        # a weight gradient: a sum over a ragged number of tokens, both sides scaled row by row, gradients with a wide exponent
        _matmul_case("matmul_weight_grad", 13824, 5120, 4016, dtype="f32", code="e5m2", block_rows=1),
        # a decoding batch at a 7B Norm exit with an 8-bit output matrix
        _logits_case("logits_8row_7b", "norm", 8, 4096, 32000, True),
        # a larger batch at a LayerNorm exit of an odd vocabulary, in bf16
        _logits_case("logits_200row_layernorm", "layernorm", 200, 4096, 32003, False),
        # one sequence being sampled: latency
        _sample_case("sample_1row", 1, 32000),
        # a serving batch of bf16 logits under a grammar's mask, an odd vocabulary
        _sample_case("sample_64row_mask", 64, 50021, dtype="bf16", mask=True),
        # a large batch of a large vocabulary, nucleus sampling alone
        _sample_case("sample_512row_nucleus", 512, 128000, filters="nucleus"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize"] * 2 + ["matmul"] * 3 + ["logits"] * 2 + ["sample"] * 3)
    if op == "quantize":
        rows, cols = _log_int(rng, 1, 32000), _log_int(rng, 64, 14000)
        rows = max(1, min(rows, 130_000_000 // cols))
        case = _quantize_case("", rows, cols, rng.choice(["bf16", "f32"]), rng.choice([1, 128]), rng.choice(["e4m3"] * 3 + ["e5m2"]),
                              rng.choice(["as_is", "as_is", "transposed", "both"]))
    elif op == "matmul":
        form = rng.choice(["decode", "decode", "batch", "weight_grad"])
        depth = 16 * _log_int(rng, 8, 900)
        features = _log_int(rng, 500, 33000)
        if form == "decode":
            case = _matmul_case("", _log_int(rng, 1, 300), features, depth, rng.choice(["bf16", "f32"]))
        else:
            rows = max(64, min(_log_int(rng, 200, 8200), int(5e11 / depth / features)))
            grad = form == "weight_grad"
            case = _matmul_case("", rows, features, depth, "f32" if grad else rng.choice(["bf16", "f32"]),
                                rng.choice(["e4m3", "e5m2"]) if grad else "e4m3", 1 if grad else 128)
    elif op == "logits":
        case = _logits_case("", rng.choice(["norm", "norm", "layernorm", "embedding"]), _log_int(rng, 1, 500), 64 * _log_int(rng, 8, 128),
                            _log_int(rng, 2000, 64000), rng.random() < 0.6, rng.choice(["bf16"] * 4 + ["f32"]))
        if case["dtype"] == "f32":
            case["scaled"] = False
    else:
        vocab = _log_int(rng, 1000, 260000)
        rows = max(1, min(_log_int(rng, 1, 1000), 60_000_000 // vocab))
        case = _sample_case("", rows, vocab, rng.choice(["f32", "bf16"]), rng.choice(["mixed", "mixed", "top_k", "nucleus", "none"]),
                            rng.random() < 0.3)
    return {k: v for k, v in case.items() if k != "name"}


# ------------------------------------------------------------ plain quantizing
def _padded(n):
    return -(-n // 16) * 16


def _plain_quantize(x, block_rows, code):
    """Codes [rows][columns padded to 16] and scales [column block][row block] of an fp32 matrix."""
    rows, cols = x.shape
    _, dtype, most = CODES[code]
    rb, cb = -(-rows // block_rows), -(-cols // BLOCK)
    x = torch.nn.functional.pad(x, (0, cb * BLOCK - cols, 0, rb * block_rows - rows)).view(rb, block_rows, cb, BLOCK)
    amax = x.abs().amax(dim=(1, 3))
    scale = torch.clamp(amax / torch.full_like(amax, most), min=LEAST)
    inverse = torch.ones_like(scale) / scale
    q = (x * inverse[:, None, :, None]).reshape(rb * block_rows, cb * BLOCK)
    return q[:rows, :_padded(cols)].to(dtype).contiguous(), scale.t().contiguous()


def _plain_values(q, scale, block_rows):
    """fp32 values of codes [rows][cols] with scales [column block][row block]."""
    s = scale.t().repeat_interleave(block_rows, 0)[:q.shape[0]].repeat_interleave(BLOCK, 1)[:, :q.shape[1]]
    return q.float() * s


# ------------------------------------------------------------------ inputs
def _rows_of(case, rows, cols, gen):
    """Activations: a scale of its own for each row."""
    x = torch.randn(rows, cols, generator=gen, device=DEVICE)
    return x.mul_(torch.exp(0.5 * torch.randn(rows, 1, generator=gen, device=DEVICE)))


def _sampling(case, gen):
    """Each row's parameters, as the requests of a batch bring them."""
    n, t = case["rows"], {}

    def pick(values):
        at = torch.randint(len(values), (n,), generator=gen, device=DEVICE)
        return torch.tensor(values, dtype=torch.float32, device=DEVICE)[at]

    t["temperature"] = pick([0.0, 0.7, 0.7, 1.0, 1.0, 1.3] if case["filters"] == "mixed" else [0.7, 1.0])
    t["top_k"] = {"mixed": [0, 1, 20, 50, 400], "top_k": [40, 50, 64]}.get(case["filters"], [0])
    t["top_k"] = pick(t["top_k"]).to(torch.int32)
    t["top_p"] = pick({"mixed": [1.0, 0.95, 0.9, 0.5], "nucleus": [0.95, 0.9, 0.8]}.get(case["filters"], [1.0]))
    t["min_p"] = pick([0.0, 0.0, 0.05] if case["filters"] == "mixed" else [0.0])
    t["uniform"] = torch.rand(n, generator=gen, device=DEVICE)
    return t


def _inputs(case, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    if case["op"] == "quantize":
        x = _rows_of(case, case["rows"], case["cols"], gen)
        return {"x": x.to(TYPES[case["dtype"]][1])}
    if case["op"] == "matmul":
        a = _rows_of(case, case["rows"], case["depth"], gen)
        b = 0.02 * torch.randn(case["features"], case["depth"], generator=gen, device=DEVICE)
        aq, sa = _plain_quantize(a, 1, case["code"])
        bq, sb = _plain_quantize(b, case["block_rows"], "e4m3")
        return {"a": aq, "a_scale": sa, "b": bq, "b_scale": sb}
    if case["op"] == "logits":
        dtype = TYPES[case["dtype"]][1]
        x = _rows_of(case, case["rows"], case["hidden"], gen)
        if case["kind"] == "layernorm":
            x += torch.randn(case["rows"], 1, generator=gen, device=DEVICE)
        t = {"x": x.to(dtype), "gamma": None, "beta": None}
        w = 0.02 * torch.randn(case["vocab"], case["hidden"], generator=gen, device=DEVICE)
        if case["kind"] != "embedding":
            t["gamma"] = (1 + 0.1 * torch.randn(case["hidden"], generator=gen, device=DEVICE)).to(dtype)
        if case["kind"] == "layernorm":
            t["beta"] = (0.1 * torch.randn(case["hidden"], generator=gen, device=DEVICE)).to(dtype)
        if case["scaled"]:
            t["w"], t["w_scale"] = _plain_quantize(w, BLOCK, "e4m3")
        else:
            t["w"] = w.to(dtype)
        return t
    n, v = case["rows"], case["vocab"]
    x = torch.randn(n, v, generator=gen, device=DEVICE).mul_(2.0 + torch.rand(n, 1, generator=gen, device=DEVICE))
    at = torch.randint(v, (n, 24), generator=gen, device=DEVICE)
    x.scatter_add_(1, at, 3 + 9 * torch.rand(n, 24, generator=gen, device=DEVICE))
    t = {"logits": x.to(TYPES[case["dtype"]][1]), "allowed": None}
    del x
    if case["mask"]:
        # what a grammar leaves differs from row to row, and may be nothing
        share = torch.tensor([0.0, 0.001, 0.1, 0.9], device=DEVICE)[torch.randint(4, (n, 1), generator=gen, device=DEVICE)]
        bits = torch.rand(n, -(-v // 32), 32, generator=gen, device=DEVICE) < share[:, :, None]
        t["allowed"] = (bits.to(torch.int64) << torch.arange(32, device=DEVICE)).sum(2).to(torch.int32)
    t.update(_sampling(case, gen))
    return t


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "quantize":
        rows, cols = case["rows"], case["cols"]
        for name, r, c in (("q", rows, cols), ("qt", cols, rows)):
            if case["out"] == "both" or (case["out"] == "as_is") == (name == "q"):
                s[name] = torch.zeros(r, _padded(c), dtype=CODES[case["code"]][1], device=DEVICE)
                s[name + "_scale"] = torch.zeros(-(-c // BLOCK), -(-r // case["block_rows"]), device=DEVICE)
    elif case["op"] == "matmul":
        s["c"] = torch.zeros(case["rows"], case["features"], dtype=TYPES[case["dtype"]][1], device=DEVICE)
    elif case["op"] == "logits":
        s["logits"] = torch.zeros(case["rows"], case["vocab"], dtype=TYPES[case["dtype"]][1], device=DEVICE)
        # room for the exit's own work: what the call asks for is asked before, once
        s["ws"] = torch.empty(64 << 20, dtype=torch.uint8, device=DEVICE)
    else:
        n = case["rows"]
        s["token"] = torch.zeros(n, dtype=torch.int32, device=DEVICE)
        s["prob"] = torch.zeros(n, device=DEVICE)
        s["confidence"] = torch.zeros(n, device=DEVICE)
        s["exit_flag"] = torch.zeros(n, dtype=torch.int32, device=DEVICE)
        s["ws"] = torch.empty(64 << 20, dtype=torch.uint8, device=DEVICE)
    return s


THRESHOLD = 0.5


# --------------------------------------------------------------- plain forms
def _plain_normed(x, gamma, beta, centre):
    if gamma is None:
        return x
    if centre:
        x = x - x.mean(dim=1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS) * gamma.float()
    return x if beta is None else x + beta.float()


def _plain_sample(s):
    x, n, v = s["logits"], s["case"]["rows"], s["case"]["vocab"]
    ids = torch.arange(v, device=x.device)
    x = x.float()
    if s["allowed"] is not None:
        bits = (s["allowed"][:, ids // 32] >> (ids % 32).to(torch.int32)) & 1
        x = torch.where(bits == 1, x, -math.inf)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    x = x.double()  # 64 bits: sums over a vocabulary, and masses next to a border
    top = x.amax(dim=1, keepdim=True)
    valid = torch.isfinite(top)
    d = x - torch.where(valid, top, 0.0)
    greedy = s["temperature"][:, None] <= 0
    mass = torch.exp(d / torch.where(greedy, 1.0, s["temperature"][:, None].double()))
    ranked = torch.gather(mass, 1, order)
    k = s["top_k"][:, None]
    keep = (ids[None] < k) | (k <= 0)
    ranked = torch.where(keep, ranked, 0.0)
    before = torch.cumsum(ranked, 1)
    p = s["top_p"][:, None].double()
    target = torch.where(p < 1, p * before[:, -1:], math.inf)
    before = torch.cat([torch.zeros_like(before[:, :1]), before[:, :-1]], 1)
    keep &= (before < target) & (ranked >= s["min_p"][:, None].double().clamp(max=1.0))
    keep &= ~greedy
    keep[:, 0] = True
    kept = torch.zeros_like(mass).scatter_(1, order, torch.where(keep, ranked, 0.0))
    upto = torch.cumsum(kept, 1)
    goal = s["uniform"][:, None].double() * upto[:, -1:]
    token = (upto <= goal).sum(1, keepdim=True).clamp(max=v - 1)
    prob = torch.gather(kept, 1, token) / upto[:, -1:]
    confidence = torch.where(valid, 1.0 / torch.exp(d).sum(1, keepdim=True), 0.0).float()
    return {"token": torch.where(valid, token, -1)[:, 0].to(torch.int32), "prob": torch.where(valid, prob, 0.0)[:, 0].float(),
            "confidence": confidence[:, 0], "exit_flag": (confidence[:, 0] > THRESHOLD).to(torch.int32)}


def _plain(s):
    case = s["case"]
    if case["op"] == "quantize":
        out = {}
        x = s["x"].float()
        for name, y in (("q", x), ("qt", x.t())):
            if name in s:
                out[name], out[name + "_scale"] = _plain_quantize(y, case["block_rows"], case["code"])
        return out
    if case["op"] == "matmul":
        c = _plain_values(s["a"], s["a_scale"], 1) @ _plain_values(s["b"], s["b_scale"], case["block_rows"]).t()
        return {"c": c.to(s["c"].dtype)}
    if case["op"] == "logits":
        z = _plain_normed(s["x"].float(), s["gamma"], s["beta"], case["kind"] == "layernorm")
        if case["scaled"]:
            q, scale = _plain_quantize(z, 1, "e4m3")
            z, w = _plain_values(q, scale, 1), _plain_values(s["w"], s["w_scale"], BLOCK)
        else:
            w = s["w"].float()
        return {"logits": (z @ w.t()).to(s["logits"].dtype)}
    return _plain_sample(s)


# ------------------------------------------------------------ the framework's
def _kernels(s):
    from paper_2402_00518_amd import binding as B

    case, stream = s["case"], torch.cuda.current_stream().cuda_stream
    if case["op"] == "quantize":
        x, br, code = s["x"], case["block_rows"], CODES[case["code"]][0]
        made = {k: B.make_scaled(s[k], s[k + "_scale"], br, code) for k in ("q", "qt") if k in s}
        B.ee_quantize_blocks(x, TYPES[case["dtype"]][0], case["rows"], case["cols"], case["cols"], made.get("q"), made.get("qt"), stream)
        return {k: s[k] for k in ("q", "q_scale", "qt", "qt_scale") if k in s}
    if case["op"] == "matmul":
        a = B.make_scaled(s["a"], s["a_scale"], 1, CODES[case["code"]][0])
        b = B.make_scaled(s["b"], s["b_scale"], case["block_rows"], B.EE_E4M3)
        B.ee_scaled_matmul(a, b, s["c"], TYPES[case["dtype"]][0], case["features"], 0, stream)
        return {"c": s["c"]}
    if case["op"] == "logits":
        dtype = TYPES[case["dtype"]][0]
        kind = B.EE_EXIT_EMBEDDING if case["kind"] == "embedding" else B.EE_EXIT_NORM
        e = B.make_exit(kind, dtype, case["hidden"], case["vocab"], 0, EPS, w_out=None if case["scaled"] else s["w"], gamma=s["gamma"],
                        beta=s["beta"], norm=B.EE_NORM_LAYER if case["kind"] == "layernorm" else B.EE_NORM_RMS)
        w = B.make_scaled(s["w"], s["w_scale"], BLOCK, B.EE_E4M3) if case["scaled"] else None
        B.ee_exit_logits(e, w, s["x"], case["rows"], s["logits"], dtype, case["vocab"], s["ws"], s["ws"].numel(), stream)
        return {"logits": s["logits"]}
    how = B.make_sampling(s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    words = 0 if s["allowed"] is None else s["allowed"].shape[1]
    B.ee_sample(s["logits"], TYPES[case["dtype"]][0], case["rows"], case["vocab"], case["vocab"], s["allowed"], words, how, s["uniform"],
                THRESHOLD, s["token"], s["prob"], s["confidence"], s["exit_flag"], s["ws"], s["ws"].numel(), stream)
    return {k: s[k] for k in ("token", "prob", "confidence", "exit_flag")}


def run(state):
    return _kernels(state) if own else _plain(state)


# -------------------------------------------------------------------- work
def work(case):
    if case["op"] == "quantize":
        r, c = case["rows"], case["cols"]
        outs = 2 if case["out"] == "both" else 1
        scales = -(-r // case["block_rows"]) * -(-c // BLOCK)
        return {"bytes": float(r * c * (TYPES[case["dtype"]][2] + outs) + 4 * outs * scales), "flops": 3.0 * r * c}
    if case["op"] == "matmul":
        m, n, k = case["rows"], case["features"], case["depth"]
        scales = -(-k // BLOCK) * (m + -(-n // case["block_rows"]))
        return {"bytes": float((m + n) * k + 4 * scales + m * n * TYPES[case["dtype"]][2]), "flops": 2.0 * m * n * k}
    if case["op"] == "logits":
        n, h, v, es = case["rows"], case["hidden"], case["vocab"], TYPES[case["dtype"]][2]
        w = v * h + 4 * -(-v // BLOCK) * -(-h // BLOCK) if case["scaled"] else v * h * es
        return {"bytes": float(n * h * es + w + n * v * es), "flops": 2.0 * n * h * v}
    n, v = case["rows"], case["vocab"]
    return {"bytes": float(n * v * TYPES[case["dtype"]][2] + (n * v / 8 if case["mask"] else 0) + 36 * n), "flops": 20.0 * n * v}


# -------------------------------------------------------- 64-bit references
def _exact_codes(x, block_rows, code):
    """Scales and codes block by block from the definition, in 64 bits."""
    rows, cols = x.shape
    most = CODES[code][2]
    scale = torch.zeros(-(-cols // BLOCK), -(-rows // block_rows), dtype=torch.float64, device=DEVICE)
    q = torch.zeros(rows, _padded(cols), dtype=torch.float64, device=DEVICE)
    for j in range(scale.shape[0]):
        part = x[:, j * BLOCK:(j + 1) * BLOCK].double()
        top = part.abs().max(dim=1).values
        if block_rows > 1:
            top = torch.stack([t.max() for t in top.split(block_rows)])
        scale[j] = torch.maximum(top / most, torch.full_like(top, LEAST))
        y = part / scale[j].repeat_interleave(block_rows)[:rows, None]
        # to the nearest code, ties to even: steps of 2^-bits relative to the power of two below
        bits, least = (3, -6) if code == "e4m3" else (2, -14)
        step = torch.exp2(torch.clamp(torch.floor(torch.log2(y.abs().clamp(min=1e-30))), min=least) - bits)
        q[:, j * BLOCK:j * BLOCK + part.shape[1]] = torch.round(y / step) * step
    return q, scale


def _exact_matrix(q, scale, block_rows):
    v = q.double()
    for j in range(scale.shape[0]):
        v[:, j * BLOCK:(j + 1) * BLOCK] *= scale[j].double().repeat_interleave(block_rows)[:v.shape[0], None]
    return v


def _exact_row(x, allowed, temperature, k, p, min_p, u):
    """(probability of the sampled token, confidence) of one row of logits."""
    if allowed is not None:
        x = x.masked_fill(~allowed, -math.inf)
    if not bool(torch.isfinite(x.max())):
        return 0.0, 0.0
    confidence = float(torch.softmax(x, 0).max())
    if temperature <= 0:
        return 1.0, confidence
    prob = torch.softmax(x / temperature, 0)
    order = torch.argsort(-x, stable=True)
    if k > 0:
        order = order[:k]
    if p < 1:
        share = torch.cumsum(prob[order], 0) / prob[order].sum()
        order = order[:int((share < p).sum()) + 1]
    order = order[prob[order] >= min(min_p, 1.0) * prob[order[0]]]
    ids = torch.sort(order).values
    kept = prob[ids] / prob[ids].sum()
    at = int(torch.searchsorted(torch.cumsum(kept, 0), u, right=True).clamp(max=len(ids) - 1))
    return float(kept[at]), confidence


def exact(case, seed):
    t = _inputs(case, seed)
    if case["op"] == "quantize":
        out = {}
        for name, x in (("q", t["x"]), ("qt", t["x"].t())):
            if case["out"] == "both" or (case["out"] == "as_is") == (name == "q"):
                out[name], out[name + "_scale"] = _exact_codes(x, case["block_rows"], case["code"])
        return out
    if case["op"] == "matmul":
        return {"c": _exact_matrix(t["a"], t["a_scale"], 1) @ _exact_matrix(t["b"], t["b_scale"], case["block_rows"]).t()}
    if case["op"] == "logits":
        z = t["x"].double()
        if t["gamma"] is not None:
            mean = z.mean(1, keepdim=True) if case["kind"] == "layernorm" else 0.0
            z = (z - mean) / ((z - mean).square().mean(1, keepdim=True) + EPS).sqrt() * t["gamma"].double()
            z = z if t["beta"] is None else z + t["beta"].double()
        if case["scaled"]:
            q, scale = _exact_codes(z, 1, "e4m3")
            return {"logits": _exact_matrix(q, scale, 1)[:, :case["hidden"]] @ _exact_matrix(t["w"], t["w_scale"], BLOCK)[:, :case["hidden"]].t()}
        return {"logits": z @ t["w"].double().t()}
    rows = []
    for i in range(case["rows"]):
        allowed = None
        if t["allowed"] is not None:
            allowed = ((t["allowed"][i][:, None] >> torch.arange(32, device=DEVICE)) & 1).bool().reshape(-1)[:case["vocab"]]
        rows.append(_exact_row(t["logits"][i].double(), allowed, *(float(t[k][i]) for k in ("temperature",)), int(t["top_k"][i]),
                               *(float(t[k][i]) for k in ("top_p", "min_p", "uniform"))))
    both = torch.tensor(rows, dtype=torch.float64, device=DEVICE)
    return {"token": None, "prob": both[:, 0], "confidence": both[:, 1], "exit_flag": None}
