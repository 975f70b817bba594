"""The operators at a pipeline's end and between its iterations, as timed cases: one pass each.

`logprob`: what a stage with the output head makes of its logits: the log probability of every row's token, the entropy of its
distribution and the likeliest alternatives, and the gradient of the logits, either in the same call (a loss, whose
weights are known before it) or in a call of its own (a policy, whose weights come from the log probabilities).  `clip`: the
norm of all gradients of a stage and the gradients scaled down to a largest norm.  `adamw`: the weights' update from
gradients whose norm is known, which takes them scaled without writing them back.

Where `own` is false a pass computes the operators from elementary torch operations in fp32 (sums over all gradients in 64
bits); where it is true it calls the kernel-level entry points of include/stage_kernels.h.  `exact` is the definition in 64 bits.
"""
import ctypes as C
import math
import random

import torch

own = False

DEV = "cuda:0"
TORCH_DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _logprob(name, **kw):
    """mode: loss (values and gradient in one call), policy (two calls) or score (values only); pad: columns between the rows; none: share of
    rows without a token; banned: share of columns whose logits are -inf."""
    return dict(dict(name=name, kind="logprob", dtype="bf16", mode="loss", pad=0, none=0.0, banned=0.0, top=0, entropy=False, scale=1.0), **kw)


def _update(name, kind, **kw):
    """flat: all tensors in one; align: elements that a tensor's start in the common buffer is a multiple of; layers of hidden x heads x ffn."""
    return dict(dict(name=name, kind=kind, dtype="bf16", grad="fp32", flat=False, align=8, bias=False), **kw)


def listed():
    return [
        # a small fp32 model whose loss a user first checks
        _logprob("loss_fp32", dtype="fp32", rows=128, vocab=1000),
        # a microbatch of a Llama-style model, a tenth of its rows masked
        _logprob("loss_layer", rows=4096, vocab=32000, none=0.1),
        # the same with a wide vocabulary: the largest case
        _logprob("loss_wide", rows=4096, vocab=128000),
        # a policy's step with a bonus on the entropy: an odd vocabulary without padding, so that rows start anywhere
        _logprob("policy_odd", mode="policy", rows=1023, vocab=50333, none=0.3, entropy=True),
        # scoring of given tokens, with the alternatives of each
        _logprob("score_top", mode="score", rows=2048, vocab=128000, top=20, entropy=True),
        # the next tokens of a few sequences at a temperature: latency
        _logprob("next_tokens", mode="score", rows=8, vocab=128000, top=20, entropy=True, scale=1.0 / 0.7, banned=0.01),
        # one token in fp32
        _logprob("next_fp32", mode="score", dtype="fp32", rows=1, vocab=32000, top=5),
        # a layer of the full-size stage, its gradients in one buffer as the stage keeps them: a fp32 accumulator of 202 million
        _update("clip_stage", "clip", layers=1, hidden=4096, heads=32, kv=32, hd=128, ffn=11008, flat=True),
        # bf16 gradients tensor by tensor, behind one another in buckets
        _update("clip_tensors", "clip", grad="bf16", layers=24, hidden=1024, heads=16, kv=4, hd=64, ffn=2816, bias=True, align=1),
        # the small fp32 stage: latency
        _update("clip_small", "clip", layers=2, hidden=256, heads=4, kv=4, hd=64, ffn=1024, bias=True),
        # the full-size layer's bf16 weights with their fp32 copies and moments
        _update("adamw_stage", "adamw", layers=1, hidden=4096, heads=32, kv=32, hd=128, ffn=11008, flat=True),
        # the small fp32 stage
        _update("adamw_small", "adamw", dtype="fp32", layers=2, hidden=256, heads=4, kv=4, hd=64, ffn=1024, bias=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    cases = listed()
    limit = max(_cost(c) for c in cases)
    # what the plain form keeps of a pass: several fp32 copies of the logits
    most = max(c["rows"] * c["vocab"] for c in cases if c["kind"] == "logprob")
    while True:
        c = _draw_one(rng)
        if _cost(c) <= limit and (c["kind"] != "logprob" or c["rows"] * c["vocab"] <= most // (1 if c["top"] == 0 else 2)):
            return c


def _cost(case):
    return work(case)["bytes"]


def _draw_one(rng):
    kind = rng.choice(["logprob", "logprob", "logprob", "logprob", "clip", "adamw"])
    if kind == "logprob":
        mode = rng.choice(["loss", "loss", "policy", "score", "score"])
        c = _logprob("", mode=mode, dtype="fp32" if rng.random() < 0.25 else "bf16", vocab=_log_int(rng, 100, 200000),
                     rows=_log_int(rng, 1, 4096) if mode == "score" else _log_int(rng, 32, 8192), none=rng.choice([0.0, 0.1, 0.5]),
                     pad=rng.choice([0, 0, rng.randrange(1, 128)]), banned=rng.choice([0.0, 0.0, 0.02, 0.5]), scale=rng.choice([1.0, 1.0, 0.5, 1.0 / 0.7]),
                     top=rng.choice([0, 1, 5, 20, 64]) if mode == "score" else 0, entropy=mode == "policy" or rng.random() < 0.4)
    else:
        hd = rng.choice([64, 128])
        heads = _log_int(rng, 1, 32)
        c = _update("", kind, dtype=rng.choice(["bf16", "bf16", "fp32"]), grad=rng.choice(["fp32", "fp32", "bf16"]), layers=_log_int(rng, 1, 16), hidden=_log_int(rng, 64, 4096),
                    heads=heads, kv=heads // rng.choice([g for g in (1, 1, 4, 8) if heads % g == 0]), hd=hd, ffn=_log_int(rng, 100, 11008),
                    flat=rng.random() < 0.3, align=rng.choice([1, 8, 8]), bias=rng.random() < 0.5)
    del c["name"]
    return c


def _tensors(case):
    """(start, size) of every tensor in the common buffer, and the buffer's size."""
    d, f, n, kv = case["hidden"], case["ffn"], case["heads"] * case["hd"], case["kv"] * case["hd"]
    layer = [d, d * (n + 2 * kv), n * d, d, d * 2 * f, f * d] + ([n + 2 * kv, d, 2 * f, d] if case["bias"] else [])
    sizes, a = layer * case["layers"], case["align"]
    if case["flat"]:
        return [(0, sum(sizes))], sum(sizes)
    out, at = [], 0
    for size in sizes:
        out.append((at, size))
        at += -(-size // a) * a
    return out, at


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype="fp32", std=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(std).to(TORCH_DTYPE[dtype])


def prepare(case, seed):
    return (_prepare_logprob if case["kind"] == "logprob" else _prepare_update)(case, seed)


def _prepare_logprob(case, seed):
    g = _gen(seed)
    rows, vocab = case["rows"], case["vocab"]
    # an offset and a spread of its own to each row: some are nearly certain, some know nothing
    std = torch.rand(rows, 1, generator=g, device=DEV) * 4.0 + 0.5
    wide = torch.randn(rows, vocab + case["pad"], generator=g, device=DEV).mul_(std).add_(_normal(g, (rows, 1), std=4.0))
    if case["banned"]:
        gone = torch.rand(vocab + case["pad"], generator=g, device=DEV) < case["banned"]
        gone[0] = False
        wide.masked_fill_(gone, -math.inf)
    wide = wide.to(TORCH_DTYPE[case["dtype"]])
    target = torch.randint(0, vocab, (rows,), generator=g, device=DEV, dtype=torch.int32)
    if case["banned"]:
        target[gone[target.long()]] = 0
    target[torch.rand(rows, generator=g, device=DEV) < case["none"]] = -1
    s = dict(case=case, logits=wide[:, :vocab], target=target, logp=torch.zeros(rows, device=DEV), stats=torch.zeros(rows, 2, device=DEV))
    if case["entropy"]:
        s["entropy"] = torch.zeros(rows, device=DEV)
    if case["top"]:
        s["top_id"] = torch.zeros(rows, case["top"], device=DEV, dtype=torch.int32)
        s["top_logp"] = torch.zeros(rows, case["top"], device=DEV)
    if case["mode"] != "score":
        s["dlogits"] = torch.zeros_like(wide)[:, :vocab]
        s["dlogp"] = torch.full((rows,), -1.0 / rows, device=DEV) if case["mode"] == "loss" else _normal(g, (rows,), std=1.0 / rows)
        if case["entropy"]:
            s["dentropy"] = torch.full((rows,), -0.01 / rows, device=DEV)
    return s


def _prepare_update(case, seed):
    g = _gen(seed)
    tensors, n = _tensors(case)
    inside = torch.ones(n, device=DEV, dtype=torch.bool)
    for (at, size), (after, _) in zip(tensors, tensors[1:] + [(n, 0)]):
        inside[at + size:after] = False

    def values(dtype, std):
        return _normal(g, (n,), dtype, std).mul_(inside)

    s = dict(case=case, tensors=tensors, grad=values(case["grad"], 0.01), max_norm=1.0)
    if case["kind"] == "clip":
        s["out"] = torch.zeros_like(s["grad"])
        s["norm"] = torch.zeros(1, device=DEV)
        s["sumsq"] = torch.zeros(1, device=DEV, dtype=torch.float64)
    else:
        s["master"] = values("fp32", 0.02)
        s["w"] = s["master"] if case["dtype"] == "fp32" else s["master"].to(torch.bfloat16)
        s["m"], s["v"] = values("fp32", 1e-3), values("fp32", 1e-3).square_()
        s["sumsq"] = s["grad"].double().square().sum().reshape(1)
        s["hyper"] = dict(lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=1 + seed % 100)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"logprob": _own_logprob, "clip": _own_clip, "adamw": _own_adamw}[kind](state)
    return {"logprob": _plain_logprob, "clip": _plain_clip, "adamw": _plain_adamw}[kind](state)


def _plain_logprob(s):
    case, scale = s["case"], s["case"]["scale"]
    x = s["logits"].float()
    top = x.amax(1)
    d = (x - top[:, None]) * scale
    e = torch.exp(d)
    total = e.sum(1)
    lnsum = torch.log(total)
    has = s["target"] >= 0
    at = s["target"].clamp(min=0).long()[:, None]
    out = dict(logp=torch.where(has, d.gather(1, at)[:, 0] - lnsum, 0.0), stats=torch.stack((top, lnsum), 1))
    if case["entropy"]:
        out["entropy"] = lnsum - torch.where(e > 0, e * d, 0.0).sum(1) / total
    if case["top"]:
        best, where = torch.sort(x, dim=1, descending=True, stable=True)
        out["top_id"] = where[:, :case["top"]].to(torch.int32)
        out["top_logp"] = (best[:, :case["top"]] - top[:, None]) * scale - lnsum[:, None]
    if case["mode"] != "score":
        p = e / total[:, None]
        w = torch.where(has, s["dlogp"], 0.0)
        grad = -w[:, None] * p
        if case["entropy"]:
            grad = grad - s["dentropy"][:, None] * torch.where(p > 0, p * (d - lnsum[:, None] + out["entropy"][:, None]), 0.0)
        grad.scatter_add_(1, at, w[:, None])
        out["dlogits"] = (grad * scale).to(s["logits"].dtype)
    return out


def _plain_clip(s):
    g = s["grad"]
    norm = g.double().square().sum().sqrt()
    coef = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0).float()
    return dict(norm=norm.float().reshape(1), out=(g.float() * coef).to(g.dtype))


def _plain_adamw(s):
    h, norm = s["hyper"], s["sumsq"].sqrt()
    g = s["grad"].float() * torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0).float()
    s["m"].mul_(h["beta1"]).add_(g * (1.0 - h["beta1"]))
    s["v"].mul_(h["beta2"]).add_(g * g * (1.0 - h["beta2"]))
    c1, c2 = 1.0 - h["beta1"] ** h["step"], 1.0 - h["beta2"] ** h["step"]
    step = (s["m"] / c1) / (torch.sqrt(s["v"] / c2) + h["eps"]) + h["weight_decay"] * s["master"]
    s["master"].sub_(h["lr"] * step)
    s["w"].copy_(s["master"])
    return dict(w=s["w"], master=s["master"], m=s["m"], v=s["v"])


# ---------------------------------------------------------------------------
# the framework's operators
# ---------------------------------------------------------------------------
def _p(t):
    return None if t is None else t.data_ptr()


def _ok(rc, what):
    if rc:
        raise RuntimeError("%s returned %d" % (what, rc))


def _own_logprob(s):
    from paper_2507_00217_amd import stage as S
    L, case, x, stream = S.lib(), s["case"], s["logits"], torch.cuda.current_stream().cuda_stream
    if "args" not in s:
        a = S.TokenLogprob(dtype=S.DTYPE[case["dtype"]], rows=case["rows"], vocab=case["vocab"], top=case["top"], scale=case["scale"], target=_p(s["target"]))
        s["args"] = a
        s["scratch"] = torch.empty(L.stage_kernel_token_logprob_scratch_bytes(C.byref(a)), dtype=torch.uint8, device=DEV)
    a = C.byref(s["args"])
    values = [_p(s["logp"]), _p(s["stats"]), _p(s.get("entropy")), _p(s.get("top_id")), _p(s.get("top_logp")), _p(s["scratch"]), s["scratch"].numel()]
    out = {n: s[n] for n in ("logp", "stats", "entropy", "top_id", "top_logp", "dlogits") if n in s}
    if case["mode"] == "loss":
        d = s["dlogits"]
        _ok(L.stage_kernel_token_logprob_grad(a, _p(x), x.stride(0), _p(s["dlogp"]), _p(s.get("dentropy")), None, _p(d), d.stride(0), *values, 0, stream),
            "stage_kernel_token_logprob_grad")
        return out
    _ok(L.stage_kernel_token_logprob_fwd(a, _p(x), x.stride(0), *values, 0, stream), "stage_kernel_token_logprob_fwd")
    if case["mode"] == "policy":
        d = s["dlogits"]
        _ok(L.stage_kernel_token_logprob_bwd(a, _p(x), x.stride(0), _p(s["stats"]), _p(s.get("entropy")), _p(s["dlogp"]), _p(s.get("dentropy")), None,
                                             _p(d), d.stride(0), 0, stream), "stage_kernel_token_logprob_bwd")
    return out


def _lists(s, *names):
    """Host arrays of the tensors' sizes, and of their addresses in each of the named buffers."""
    n = len(s["tensors"])
    if "sizes" not in s:
        s["sizes"] = (C.c_int64 * n)(*[size for _, size in s["tensors"]])
        s["lists"] = {k: (C.c_void_p * n)(*[s[k].data_ptr() + at * s[k].element_size() for at, _ in s["tensors"]]) for k in names}
    return [n, s["sizes"]] + [s["lists"][k] for k in names]


def _own_clip(s):
    from paper_2507_00217_amd import stage as S
    L, dt, stream = S.lib(), S.DTYPE[s["case"]["grad"]], torch.cuda.current_stream().cuda_stream
    n, sizes, grads, outs = _lists(s, "grad", "out")
    if "scratch" not in s:
        s["scratch"] = torch.empty(L.stage_kernel_grad_sumsq_scratch_bytes(), dtype=torch.uint8, device=DEV)
    _ok(L.stage_kernel_grad_sumsq(dt, n, sizes, grads, 0, _p(s["sumsq"]), _p(s["scratch"]), s["scratch"].numel(), stream), "stage_kernel_grad_sumsq")
    _ok(L.stage_kernel_grad_clip(dt, n, sizes, grads, outs, _p(s["sumsq"]), s["max_norm"], _p(s["norm"]), stream), "stage_kernel_grad_clip")
    return dict(norm=s["norm"], out=s["out"])


def _own_adamw(s):
    from paper_2507_00217_amd import stage as S
    L, case = S.lib(), s["case"]
    wide = case["dtype"] == "fp32"
    n, sizes, w, master, m, v, grads = _lists(s, "w", "master", "m", "v", "grad")
    if "args" not in s:
        s["args"] = S.AdamW(dtype=S.DTYPE[case["dtype"]], grad_dtype=S.DTYPE[case["grad"]], sumsq=_p(s["sumsq"]), max_norm=s["max_norm"], **s["hyper"])
    _ok(L.stage_kernel_adamw(C.byref(s["args"]), n, sizes, w, None if wide else master, m, v, grads, torch.cuda.current_stream().cuda_stream),
        "stage_kernel_adamw")
    return dict(w=s["w"], master=s["master"], m=s["m"], v=s["v"])


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    if case["kind"] == "logprob":
        es, n, rows = 4 if case["dtype"] == "fp32" else 2, case["rows"] * case["vocab"], case["rows"]
        # logits and targets in, log probabilities and statistics out; alternatives; weights in and the gradient out.  A policy's gradient has to
        # read the logits a second time: its weights are made from what the first pass gives.
        moved = {"loss": 2, "policy": 3, "score": 1}[case["mode"]] * es * n + 16 * rows + 8 * rows * case["top"] + (4 * rows if case["entropy"] else 0)
        flops = (5.0 + (2.0 if case["entropy"] else 0.0) + (1.0 if case["top"] else 0.0) + (4.0 if case["mode"] != "score" else 0.0)) * n
        return {"bytes": moved + (8 * rows if case["mode"] != "score" else 0), "flops": flops}
    n = sum(size for _, size in _tensors(case)[0])
    eg, ew = (4 if case[x] == "fp32" else 2 for x in ("grad", "dtype"))
    if case["kind"] == "clip":
        # every gradient in for the norm, and in and out to be scaled by it
        return {"bytes": 3 * eg * n + 8, "flops": 3.0 * n}
    # gradient in, fp32 weight and moments in and out, a bf16 weight out
    return {"bytes": (eg + 24 + (2 if ew == 2 else 0)) * n, "flops": 14.0 * n}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    return {"logprob": _exact_logprob, "clip": _exact_clip, "adamw": _exact_adamw}[case["kind"]](case, seed)


def _exact_logprob(case, seed):
    s = _prepare_logprob(case, seed)
    rows, block = case["rows"], max(1, (1 << 26) // case["vocab"])
    parts = [_exact_rows(case, {k: v[i:i + block] for k, v in s.items() if k != "case"}) for i in range(0, rows, block)]
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_rows(case, s):
    """By log-sum-exp, the entropy from the probabilities' logarithms, and the gradient by differentiation of the loss."""
    x = s["logits"].double()
    keep = torch.isfinite(x)
    leaf = x.masked_fill(~keep, 0.0).requires_grad_(case["mode"] != "score")
    y = (leaf * case["scale"]).masked_fill(~keep, -math.inf)
    lse = torch.logsumexp(y, 1)
    logq = torch.where(keep, y - lse[:, None], 0.0)
    has = s["target"] >= 0
    rows = torch.arange(x.shape[0], device=DEV)
    logp = torch.where(has, logq[rows, s["target"].clamp(min=0).long()], 0.0)
    top = x.amax(1)
    out = dict(logp=logp.detach(), stats=torch.stack((top, (lse - case["scale"] * top).detach()), 1))
    entropy = -(torch.where(keep, torch.exp(logq), 0.0) * logq).sum(1)
    if case["entropy"]:
        out["entropy"] = entropy.detach()
    if case["top"]:
        best, where = torch.sort(x, dim=1, descending=True, stable=True)
        out["top_id"] = where[:, :case["top"]].to(torch.int32)
        out["top_logp"] = best[:, :case["top"]] * case["scale"] - lse[:, None]
    if case["mode"] != "score":
        loss = (logp * s["dlogp"].double()).sum()
        if case["entropy"]:
            loss = loss + (entropy * s["dentropy"].double()).sum()
        out["dlogits"] = torch.autograd.grad(loss, leaf)[0]
    return out


def _exact_clip(case, seed):
    s = _prepare_update(case, seed)
    g = s["grad"].double()
    norm = torch.linalg.vector_norm(g)
    return dict(norm=norm.reshape(1), out=g * min(1.0, s["max_norm"] / float(norm)))


def _exact_adamw(case, seed):
    s = _prepare_update(case, seed)
    h, g = s["hyper"], s["grad"].double()
    g *= min(1.0, s["max_norm"] / float(torch.linalg.vector_norm(g)))
    m = torch.lerp(s["m"].double(), g, 1.0 - h["beta1"])
    v = torch.lerp(s["v"].double(), g ** 2, 1.0 - h["beta2"])
    w = s["master"].double() * (1.0 - h["lr"] * h["weight_decay"])
    w = w - h["lr"] * (m / (1.0 - h["beta1"] ** h["step"])) / ((v / (1.0 - h["beta2"] ** h["step"])) ** 0.5 + h["eps"])
    return dict(w=w, master=w, m=m, v=v)
