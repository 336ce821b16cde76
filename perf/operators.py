"""The 8-bit projections and the scoring of tokens, as cases to be timed and compared.

A case is one call:

  norm      residual addition, RMSNorm, int8 rows with a scale each (`ssm_norm_i8`)
  quant     rows to int8 with a scale each, plain or through SwiGLU (`ssm_quant_i8`)
  gemm      product of int8 rows with int8 weights, scaled (`ssm_gemm_i8`)
  logprobs  log probabilities of given tokens, entropy, top alternatives (`ssm_token_logprobs`)

Shapes are those of the repository's own configurations (8B: width 4096, feed-forward 12288,
vocabulary 126464; 7B: 3584, 18944, 152064; small: 128, 512) at its steps' row counts.
8-bit outputs are returned as the values they stand for, rounded to bfloat16.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def listed():
    return [
        # One row of the 8B model: latency only.
        dict(name="norm_1x4096", kind="norm", rows=1, d=4096, delta="bf16", gain="bf16"),
        # The norm after the output projection of a block-start step, batch 8 of 1776 rows.
        dict(name="norm_14208x4096", kind="norm", rows=14208, d=4096, delta="f32", gain="bf16"),
        # SwiGLU into the down projection of a cached step: 240 rows of [gate | up].
        dict(name="quant_swiglu_240x12288", kind="quant", rows=240, d=12288, dtype="bf16", swiglu=True),
        # The attention output of a step of the 7B model before its output projection, float32.
        dict(name="quant_5081x3584", kind="quant", rows=5081, d=3584, dtype="f32", swiglu=False),
        # One row through an output projection: the weights' bytes and latency.
        dict(name="gemm_1x4096x4096", kind="gemm", rows=1, n=4096, k=4096, out="bf16"),
        # Gate and up of a cached step of 120 rows.
        dict(name="gemm_120x24576x4096", kind="gemm", rows=120, n=24576, k=4096, out="bf16"),
        # The down projection of a cached step of 240 rows.
        dict(name="gemm_240x4096x12288", kind="gemm", rows=240, n=4096, k=12288, out="f32"),
        # The down projection of the 7B model at an odd row count.
        dict(name="gemm_1127x3584x18944", kind="gemm", rows=1127, n=3584, k=18944, out="bf16"),
        # Gate and up of a cached step of a batch of 32: 3840 rows.
        dict(name="gemm_3840x24576x4096", kind="gemm", rows=3840, n=24576, k=4096, out="bf16"),
        # One row over the largest vocabulary.
        dict(name="logprobs_1x152064", kind="logprobs", rows=1, vocab=152064, dtype="f32", targets=1, k=5),
        # The output rows of a cached step: block and retained suffix.
        dict(name="logprobs_120x126464", kind="logprobs", rows=120, vocab=126464, dtype="f32", targets=1, k=5),
        # Scoring whole sequences: 3840 rows of an 8-bit head's bfloat16 logits, two tokens a row.
        dict(name="logprobs_3840x126464", kind="logprobs", rows=3840, vocab=126464, dtype="bf16", targets=2, k=8),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "quant", "gemm", "gemm", "gemm", "logprobs", "logprobs"])
    if kind == "norm":
        d = rng.choice([128, 512, 3584, 4096, _log(rng, 100, 8000)])
        return dict(kind="norm", rows=_log(rng, 1, 14208 * 4096 // max(d, 4096)), d=d,
                    delta=rng.choice(["none", "f32", "bf16", "f16"]), gain=rng.choice(["f32", "bf16"]))
    if kind == "quant":
        d = rng.choice([128, 3584, 4096, 12288, 18944, _log(rng, 100, 20000)])
        return dict(kind="quant", rows=_log(rng, 1, 5081 * 3584 // max(d, 3584)), d=d,
                    dtype=rng.choice(["f32", "bf16", "f16"]), swiglu=rng.random() < 0.5)
    if kind == "gemm":
        n, k = rng.choice([(12288, 4096), (4096, 4096), (24576, 4096), (4096, 12288), (4608, 3584),
                           (3584, 3584), (37888, 3584), (3584, 18944), (126464, 4096),
                           (_log(rng, 64, 9000), 16 * _log(rng, 8, 600)),
                           (_log(rng, 64, 4000), _log(rng, 100, 6000))])
        return dict(kind="gemm", rows=_log(rng, 1, max(1, min(4336, 3840 * 24576 * 4096 // (n * k)))), n=n, k=k,
                    out=rng.choice(["f32", "bf16", "f16"]))
    vocab = rng.choice([512, 126464, 126464, 152064, _log(rng, 300, 200000)])
    return dict(kind="logprobs", rows=_log(rng, 1, min(8000, 3840 * 126464 // vocab)), vocab=vocab,
                dtype=rng.choice(["f32", "bf16", "f16"]), targets=rng.randrange(1, 4), k=rng.randrange(1, 9))


# ---- inputs -----------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7FFFFFFF)
    return g


def _normal(g, size, std=1.0, dtype=torch.float32, mean=0.0):
    x = torch.empty(size, dtype=torch.float32, device=DEV)
    return x.normal_(mean, std, generator=g).to(dtype)


def _empty(size, dtype):
    return torch.empty(size, dtype=dtype, device=DEV)


def _inputs(case, seed):
    g, rows = _gen(seed), case["rows"]
    if case["kind"] == "norm":
        # a residual stream whose rows differ in size, as they do over depth
        d = case["d"]
        x = _normal(g, (rows, d)) * torch.exp(_normal(g, (rows, 1), 0.5))
        delta = None if case["delta"] == "none" else _normal(g, (rows, d), 0.3, DTYPES[case["delta"]])
        return dict(x=x, delta=delta, gain=_normal(g, (d,), 0.1, DTYPES[case["gain"]], 1.0))
    if case["kind"] == "quant":
        width = 2 * case["d"] if case["swiglu"] else case["d"]
        return dict(x=_normal(g, (rows, width), 1.5, DTYPES[case["dtype"]]))
    if case["kind"] == "gemm":
        n, k = case["n"], case["k"]

        def codes(r):   # normal values quantised with a row maximum of four deviations
            q = torch.empty((r, k), dtype=torch.float16, device=DEV).normal_(0.0, 127 / 4, generator=g)
            return q.round_().clamp_(-127, 127).to(torch.int8)
        return dict(a=codes(rows), w=codes(n),
                    sa=torch.exp(_normal(g, (rows,), 0.5)) * (4 / 127),
                    sw=torch.exp(_normal(g, (n,), 0.2)) * (0.08 / 127))
    vocab = case["vocab"]
    logits = _normal(g, (rows, vocab), 2.0, DTYPES[case["dtype"]])
    ids = torch.randint(0, vocab - 1, (rows, case["targets"]), generator=g, device=DEV, dtype=torch.int32)
    # a model is sure of some of its tokens: their rows peak at the first target
    sure = torch.rand((rows,), generator=g, device=DEV) < 0.5
    lift = torch.where(sure, 14.0, 3.0).to(logits.dtype)
    logits[torch.arange(rows, device=DEV), ids[:, 0].long()] += lift
    return dict(logits=logits, ids=ids, mask_id=vocab - 1, k=case["k"])


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"], rows, i8, f32 = case, case["rows"], torch.int8, torch.float32
    # output buffers, as a serving program keeps them
    if case["kind"] in ("norm", "quant"):
        d = case["d"]
        s |= dict(q=_empty((rows, d), i8), scale=_empty((rows,), f32), value=_empty((rows, d), torch.bfloat16))
        if case["kind"] == "norm":
            s["resid"] = _empty((rows, d), f32)
    elif case["kind"] == "gemm":
        s["out"] = _empty((rows, case["n"]), DTYPES[case["out"]])
    else:
        s |= dict(lp=_empty((rows, case["targets"]), f32), entropy=_empty((rows,), f32),
                  top_ids=_empty((rows, case["k"]), torch.int32), top_lp=_empty((rows, case["k"]), f32))
    if own:     # and the workspaces of the calls that take one
        from paper_2608_23167_amd import api
        if case["kind"] == "gemm":
            s["ws"] = _empty((api.ssm_gemm_i8_workspace_size(rows, case["n"], case["k"]),), torch.uint8)
        elif case["kind"] == "logprobs":
            s["ws"] = _empty((api.ssm_token_logprobs_workspace_size(rows, case["vocab"], case["k"]),), torch.uint8)
    return s


# ---- one pass ---------------------------------------------------------------
def _own(s):
    from paper_2608_23167_amd import api
    kind = s["case"]["kind"]
    if kind == "norm":
        api.ssm_norm_i8(s["x"], s["gain"], EPS, s["q"], s["scale"], delta=s["delta"], resid=s["resid"])
        return [torch.mul(s["q"], s["scale"][:, None], out=s["value"]), s["scale"], s["resid"]]
    if kind == "quant":
        api.ssm_quant_i8(s["x"], s["q"], s["scale"], swiglu=s["case"]["swiglu"])
        return [torch.mul(s["q"], s["scale"][:, None], out=s["value"]), s["scale"]]
    if kind == "gemm":
        api.ssm_gemm_i8(s["a"], s["sa"], s["w"], s["sw"], s["out"], s["ws"])
        return s["out"]
    api.ssm_token_logprobs(s["logits"], s["ids"], s["mask_id"], s["k"], s["lp"], s["entropy"],
                           s["top_ids"], s["top_lp"], s["ws"])
    return [s["lp"], s["entropy"], s["top_ids"], s["top_lp"]]


def _codes(y):
    scale = y.abs().amax(1) / 127
    q = torch.where(scale[:, None] > 0, y / scale[:, None], 0.0).round()
    return (q * scale[:, None]).to(torch.bfloat16), scale


def _logprobs(s):
    x = s["logits"].to(torch.float32, copy=True)
    x[:, s["mask_id"]] = -math.inf
    m = x.amax(1, keepdim=True)
    z = x - m
    e = z.exp()
    total = e.sum(1, keepdim=True)
    log_total = total.log()
    # sum of e * z, where z = -inf adds nothing
    entropy = log_total[:, 0] - (e * z.clamp_min(-1e30)).sum(1) / total[:, 0]
    lp = z.gather(1, s["ids"].long()) - log_total
    # the k largest, the lower id first where two are equal: the order of the float's bits above that of the ids
    bits = (x + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    key = bits * 2 ** 32 + (x.shape[1] - 1 - torch.arange(x.shape[1], device=x.device))
    top = key.topk(s["k"], dim=1, sorted=True).values
    top_ids = x.shape[1] - 1 - (top & 0xFFFFFFFF)
    return [lp, entropy, top_ids.int(), z.gather(1, top_ids) - log_total]


def run(state):
    if own:
        return _own(state)
    s, kind = state, state["case"]["kind"]
    if kind == "norm":
        r = s["x"] if s["delta"] is None else s["x"] + s["delta"].float()
        y = r * torch.rsqrt(r.square().mean(1, keepdim=True) + EPS) * s["gain"].float()
        return [*_codes(y), r]
    if kind == "quant":
        y = s["x"].float()
        if s["case"]["swiglu"]:
            gate, up = y.chunk(2, dim=1)
            y = gate / (1 + (-gate).exp()) * up
        return list(_codes(y))
    if kind == "gemm":
        acc = s["a"].float() @ s["w"].float().t()
        return (acc * s["sa"][:, None] * s["sw"]).to(s["out"].dtype)
    return _logprobs(s)


# ---- the definition in 64 bits ------------------------------------------------
def _exact_codes(y):
    largest = y.abs().max(dim=1).values
    step = torch.where(largest > 0, largest / 127, 1.0)
    code = torch.round(y / step.unsqueeze(1)).clamp(-127, 127)
    return [code * step.unsqueeze(1), largest / 127]


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "norm":
        r = s["x"].double()
        if s["delta"] is not None:
            r = r + s["delta"].double()
        rms = (torch.linalg.vector_norm(r, dim=1) ** 2 / case["d"] + EPS).sqrt()
        return _exact_codes(s["gain"].double() * r / rms.unsqueeze(1)) + [r]
    if case["kind"] == "quant":
        y = s["x"].double()
        if case["swiglu"]:
            gate, up = y[:, :case["d"]], y[:, case["d"]:]
            y = gate * torch.sigmoid(gate) * up
        return _exact_codes(y)
    if case["kind"] == "gemm":
        parts = []
        for lo in range(0, case["n"], 8192):
            hi = min(lo + 8192, case["n"])
            p = torch.mm(s["a"].double(), s["w"][lo:hi].double().t())
            parts.append(p * torch.outer(s["sa"].double(), s["sw"][lo:hi].double()))
        return torch.cat(parts, dim=1)
    outs, step = [], max(1, 2 ** 26 // case["vocab"])
    for lo in range(0, case["rows"], step):
        x = s["logits"][lo:lo + step].double()
        x[:, s["mask_id"]] = -math.inf
        logp = torch.log_softmax(x, dim=1)
        plogp = torch.where(logp > -math.inf, logp.exp() * logp, 0.0)
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["k"]]
        outs.append((logp.gather(1, s["ids"][lo:lo + step].long()), -plogp.sum(1), order.int(),
                     logp.gather(1, order)))
    return [torch.cat(part) for part in zip(*outs)]


# ---- what a pass cannot do without --------------------------------------------
def work(case):
    size = {"none": 0, "f32": 4, "bf16": 2, "f16": 2}
    rows = case["rows"]
    if case["kind"] == "norm":
        n = rows * case["d"]
        return {"bytes": n * (4 + size[case["delta"]] + 4 + 1) + case["d"] * size[case["gain"]] + rows * 4,
                "flops": 8 * n}
    if case["kind"] == "quant":
        n = rows * case["d"]
        return {"bytes": n * (size[case["dtype"]] * (2 if case["swiglu"] else 1) + 1) + rows * 4,
                "flops": (8 if case["swiglu"] else 3) * n}
    if case["kind"] == "gemm":
        n, k = case["n"], case["k"]
        return {"bytes": (rows + n) * (k + 4) + rows * n * size[case["out"]], "flops": 2 * rows * n * k}
    vocab = case["vocab"]
    return {"bytes": rows * (vocab * size[case["dtype"]] + 8 * case["targets"] + 4 + 8 * case["k"]),
            "flops": 4 * rows * vocab}
