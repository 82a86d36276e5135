"""The operators around a teacher that serves its scores, as cases that can be timed and compared.

On-policy distillation needs from the teacher the log probabilities of the student's tokens, how sure
it was (entropy) and its few most likely alternatives; a student then learns from that short list
alone.  The teacher is frozen, so its output embedding can be kept in 8 bits.

Paths (``case["path"]``):
  logprobs       logits -> log probability of each given token, entropy, log-sum-exp, the top
                 alternatives with their log probabilities, and the log of the mass outside them
  logprobs_grad  the gradient of any loss of those scores with respect to the logits
  topk_kl        divergence of the student from a teacher known by its top alternatives and the mass
                 outside them: value, sampled cost, squared gradient norm, gradient
  linear_i8      hidden states -> 8 bits per token -> product with an 8-bit output embedding -> logits

``run`` computes a path in plain torch operations where ``own`` is false, through the public binding
where it is true.  Sizes and value distributions are those of the repository's own workloads
(``synth.CONFIGS``, ``synth.LMHEAD``, the tests and the benchmark) and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# Value recipes: standard deviation of the student logits, teacher = mix * student + noise, share of
# +10 spikes (the recipes of the configs with 4 096, 32 000 and 151 936 entries).
_RECIPES = {
    "plain": dict(s_std=2.0, mix=1.0, t_std=1.0, spike_p=0.0),
    "mixed": dict(s_std=3.0, mix=0.8, t_std=1.5, spike_p=0.0),
    "spiky": dict(s_std=4.0, mix=1.0, t_std=2.0, spike_p=0.05),
}
_CHUNK = 1 << 25      # entries of a block of rows that the plain forms work on at a time
REST_FLOOR = 2.0 ** -24


def _rows_case(name, path, B, T, V, *, dtype="bf16", K=0, recipe="spiky", lo=0.25, hi=1.0,
               rollout=1.0, masked=0.0, entropy=True, mode="reverse", rest=True, ld=0):
    """Windows are spread evenly over [lo, hi] of T, rollouts over [rollout, 1] of T (a rollout
    shorter than its window ends it early).  masked: share of the vocabulary a grammar rules out."""
    return dict(name=name, path=path, B=B, T=T, V=V, ld=ld or V, dtype=dtype, K=K, recipe=recipe,
                lo=lo, hi=hi, rollout=rollout, masked=masked, entropy=entropy, mode=mode, rest=rest)


def _linear_case(name, M, V, d, *, out="bf16", w_std=0.02):
    return dict(name=name, path="linear_i8", M=M, V=V, d=d, out=out, w_std=w_std)


def listed():
    return [
        # one decoding step of 8 sequences: the teacher scores the token just sampled
        _rows_case("logprobs_token_152k", "logprobs", 8, 1, 151936, K=20, lo=1.0),
        # the prefix windows of a batch of rollouts, the largest vocabulary in use
        _rows_case("logprobs_rollouts_152k", "logprobs", 8, 1024, 151936, K=20),
        # a longer list for a student that learns from it
        _rows_case("logprobs_top64_32k", "logprobs", 8, 1024, 32000, K=64, recipe="mixed"),
        # fp32 logits of a vocabulary that is no multiple of anything, rows packed, a grammar mask
        _rows_case("logprobs_fp32_odd", "logprobs", 8, 256, 50257, dtype="f32", K=5, recipe="mixed",
                   masked=0.3, rollout=0.5),
        # policy-gradient step with an entropy bonus on the same rollouts
        _rows_case("grad_rollouts_152k", "logprobs_grad", 8, 1024, 151936),
        # fp32, packed odd rows, a loss of the alternatives' scores as well
        _rows_case("grad_fp32_odd", "logprobs_grad", 8, 256, 50257, dtype="f32", K=5,
                   recipe="mixed", rollout=0.5),
        # a unit-test-sized update in fp32: launches and host work decide
        _rows_case("topk_kl_small", "topk_kl", 2, 64, 4096, dtype="f32", K=8, recipe="plain", lo=0.5),
        # the update on the prefix windows, teacher known by 64 alternatives and the mass outside
        _rows_case("topk_kl_152k", "topk_kl", 8, 1024, 151936, K=64),
        # packed odd rows, the forward divergence, a served teacher that gives only its list
        _rows_case("topk_kl_odd", "topk_kl", 8, 512, 50257, K=20, recipe="mixed", rollout=0.5,
                   mode="forward", rest=False),
        # teacher logits of one decoding step of 8 sequences
        _linear_case("linear_i8_token", 8, 151936, 2560),
        # teacher logits of a block of rollout positions
        _linear_case("linear_i8_rollouts", 4096, 151936, 2560),
        # sizes that are no multiple of a tile, fp32 logits
        _linear_case("linear_i8_odd", 777, 50257, 1000, out="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    path = rng.choice(["logprobs"] * 4 + ["logprobs_grad"] * 3 + ["topk_kl"] * 4 + ["linear_i8"] * 3)
    if path == "linear_i8":
        V, d = _log_int(rng, 1000, 151936), _log_int(rng, 64, 2560)
        if rng.random() < 0.5:
            V, d = max(64, V // 64 * 64), max(64, d // 64 * 64)
        case = _linear_case("", _log_int(rng, 1, 4096), V, d, out=rng.choice(["bf16", "bf16", "f32"]))
        del case["name"]
        return case
    V = _log_int(rng, 1000, 151936)
    kind = rng.choice(["round", "round", "padded", "odd"])
    if kind == "round":
        V = V // 64 * 64
    ld = (V + 63) // 64 * 64 if kind == "padded" else V
    dtype = rng.choice(["bf16", "bf16", "f32"])
    rows = _log_int(rng, 1, min(16384, 6e8 / V / (2 if dtype == "f32" else 1)))
    B = min(rng.randint(1, 16), rows)
    K = _log_int(rng, 1, 128)
    if path != "topk_kl" and rng.random() < 0.2:
        K = 0
    case = _rows_case("", path, B, rows // B, V, ld=ld, dtype=dtype, K=K,
                      recipe=rng.choice(["plain", "mixed", "spiky"]),
                      lo=rng.choice([1 / 16, 0.25, 1.0]), hi=1.0, rollout=rng.choice([1.0, 0.5]),
                      masked=rng.choice([0.0, 0.0, 0.3]), entropy=rng.random() < 0.7,
                      mode=rng.choice(["reverse", "reverse", "forward"]), rest=rng.random() < 0.6)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """Window and rollout lengths as host lists (the same for every seed, so that the work is)."""
    B, T = case["B"], case["T"]

    def spread(lo, hi, order):
        step = [(b * order + order // 2) % B / max(1, B - 1) for b in range(B)] if B > 1 else [1.0]
        return [min(T, max(1, int(round(T * (lo + (hi - lo) * f))))) for f in step]

    return spread(case["lo"], case["hi"], 1), spread(case["rollout"], 1.0, 3)


def _ends(case):
    return [min(w, r) for w, r in zip(*_lengths(case))]


def _generator(seed, b):
    g = torch.Generator(device="cuda")
    g.manual_seed(1 + 104729 * int(seed) + 17 * b)
    return g


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _draw_rows(case, n, g, want_teacher):
    """n rows of student logits (fp32, not yet rounded), and of teacher logits."""
    r, V = _RECIPES[case["recipe"]], case["V"]
    z = torch.randn((n, V), generator=g, device="cuda") * r["s_std"]
    if r["spike_p"] > 0:
        z += 10.0 * (torch.rand((n, V), generator=g, device="cuda") < r["spike_p"])
    u = None
    if want_teacher:
        u = r["mix"] * z + r["t_std"] * torch.randn((n, V), generator=g, device="cuda")
    if case["masked"] > 0:
        out = torch.rand((n, V), generator=g, device="cuda") < case["masked"]
        out[:, :256] = False          # (a grammar always leaves a choice)
        z.masked_fill_(out, -math.inf)
        if u is not None:
            u.masked_fill_(out, -math.inf)
    return z, u


def _gumbel_argmax(z, g):
    e = torch.rand(z.shape, generator=g, device="cuda").clamp_(min=1e-20)
    return (z - e.log_().neg_().log_()).argmax(dim=1).int()


def prepare(case, seed):
    if case["path"] == "linear_i8":
        return _prepare_linear(case, seed)
    B, T, V, ld, K = case["B"], case["T"], case["V"], case["ld"], case["K"]
    dt = _DTYPES[case["dtype"]]
    window, rollout = _lengths(case)
    ends = _ends(case)
    logits = torch.zeros((B, T, ld), dtype=dt, device="cuda")[:, :, :V]
    tokens = torch.zeros((B, T), dtype=torch.int32, device="cuda")
    state = dict(case=case, logits=logits, tokens=tokens, window=_int32(window),
                 rollout=_int32(rollout), rows=_row_list(ends), status=_int32([0]))
    path = case["path"]
    with_list = K > 0 and path != "logprobs"
    if with_list:
        state["top_ids"] = torch.full((B, T, K), -1, dtype=torch.int32, device="cuda")
        state["top_logprobs"] = torch.zeros((B, T, K), device="cuda")
        state["rest"] = torch.zeros((B, T), device="cuda")
    if path == "logprobs_grad":
        state["lse"] = torch.zeros((B, T), device="cuda")
        state["entropy"] = torch.zeros((B, T), device="cuda")
    step = max(1, _CHUNK // V)
    for b in range(B):
        g = _generator(seed, b)
        for t0 in range(0, ends[b], step):
            t1 = min(ends[b], t0 + step)
            z, u = _draw_rows(case, t1 - t0, g, path == "topk_kl")
            z = z.to(dt)
            logits[b, t0:t1] = z
            z = z.float()
            tokens[b, t0:t1] = _gumbel_argmax(z, g)
            if with_list:      # the served list: of the teacher, or of the policy itself
                v = (z if u is None else u.to(dt).float()).double()
                lq = torch.log_softmax(v, dim=1)
                top = lq.topk(K, dim=1)
                state["top_ids"][b, t0:t1] = top.indices.int()
                state["top_logprobs"][b, t0:t1] = top.values.float()
                left = lq.exp().scatter_(1, top.indices, 0.0).sum(dim=1)
                state["rest"][b, t0:t1] = left.log().float()
                del v, lq
            if path == "logprobs_grad":
                lp = torch.log_softmax(z.double(), dim=1)
                state["lse"][b, t0:t1] = torch.logsumexp(z.double(), dim=1).float()
                state["entropy"][b, t0:t1] = -torch.where(lp > -math.inf, lp.exp() * lp, 0.0).sum(dim=1).float()
                del lp
    if path == "logprobs_grad":     # what a policy-gradient loss hands back: one weight a token
        g = _generator(seed, 998)
        state["d_logprob"] = torch.randn((B, T), generator=g, device="cuda")
        state["d_entropy"] = torch.rand((B, T), generator=g, device="cuda") * 0.1 if case["entropy"] else None
        state["d_top"] = torch.randn((B, T, K), generator=g, device="cuda") / K if K else None
    if path != "logprobs":
        state["grad"] = torch.zeros((B, T, ld), dtype=dt, device="cuda")[:, :, :V]
    return state


def _prepare_linear(case, seed):
    M, V, d = case["M"], case["V"], case["d"]
    g = _generator(seed, 0)
    hidden = torch.randn((M, d), generator=g, device="cuda").bfloat16()
    wq = torch.zeros((V, (d + 15) // 16 * 16), dtype=torch.int8, device="cuda")
    w_scale = torch.empty(V, device="cuda")
    for v0 in range(0, V, 16384):       # the frozen embedding is laid out once
        w = torch.randn((min(V, v0 + 16384) - v0, d), generator=g, device="cuda") * case["w_std"]
        q, s = _quantize(w.bfloat16())
        wq[v0:v0 + w.shape[0], :d] = q.to(torch.int8)
        w_scale[v0:v0 + w.shape[0]] = s
    return dict(case=case, hidden=hidden, wq=wq[:, :d], w_scale=w_scale,
                logits=torch.zeros((M, V), dtype=_DTYPES[case["out"]], device="cuda"), status=_int32([0]))


def _row_list(ends):
    """[(sequence, first, last + 1)] of the processed positions."""
    return [(b, 0, e) for b, e in enumerate(ends) if e > 0]


def work(case):
    if case["path"] == "linear_i8":
        M, V, d = case["M"], case["V"], case["d"]
        return {"bytes": 2 * M * d + V * d + 4 * V + M * V * (2 if case["out"] == "bf16" else 4),
                "flops": 2 * M * V * d}
    n, V, K = sum(_ends(case)), case["V"], case["K"]
    es = 2 if case["dtype"] == "bf16" else 4
    if case["path"] == "logprobs":
        return {"bytes": n * (V * es + 4 + 16 + 8 * K), "flops": 5 * n * V}
    if case["path"] == "logprobs_grad":
        return {"bytes": n * (2 * V * es + 16 + 8 * K), "flops": 5 * n * V}
    return {"bytes": n * (2 * V * es + 20 + 8 * K), "flops": 7 * n * V}


# ------------------------------------------------------------------------------------------- run
def run(state):
    path = state["case"]["path"]
    return (_OWN if own else _PLAIN)[path](state)


def _own_logprobs(s):
    from paper_2605_28396_b200 import api
    o = api.adwin_token_logprobs(s["logits"], s["tokens"], s["window"], s["rollout"],
                                 top_k=s["case"]["K"], want_entropy=s["case"]["entropy"],
                                 dev_status=s["status"])
    return _scores(o.logprob, o.entropy, o.lse, o.top_ids, o.top_logprobs, o.rest)


def _own_grad(s):
    from paper_2605_28396_b200 import api
    o = api.adwin_token_logprobs_bwd(s["logits"], s["tokens"], s["lse"], s["window"], s["rollout"],
                                     d_logprob=s["d_logprob"], d_entropy=s["d_entropy"],
                                     entropy=s["entropy"] if s["d_entropy"] is not None else None,
                                     top_ids=s.get("top_ids"), d_top=s["d_top"], grad=s["grad"],
                                     dev_status=s["status"])
    return dict(grad=o.grad)


def _own_topk_kl(s):
    from paper_2605_28396_b200 import api
    c = s["case"]
    o = api.adwin_opd_topk_kl_fwd_bwd(s["logits"], s["tokens"], s["top_ids"], s["top_logprobs"],
                                      s["window"], s["rollout"], rest=s["rest"] if c["rest"] else None,
                                      kl_mode=api.KL_FORWARD if c["mode"] == "forward" else api.KL_REVERSE,
                                      grad=s["grad"], want_lse=True, dev_status=s["status"])
    return dict(kl=o.kl, logratio=o.logratio, gsq=o.gsq, lse=o.lse_s, grad=o.grad)


def _own_linear(s):
    from paper_2605_28396_b200 import api
    q, scale = api.adwin_quantize_rows_i8(s["hidden"], dev_status=s["status"])
    out = api.adwin_linear_i8(q, scale, s["wq"], s["w_scale"], out=s["logits"], dev_status=s["status"])
    return dict(logits=out, scale=scale)


def _scores(logprob, entropy, lse, top_ids, top_logprobs, rest):
    out = dict(logprob=logprob, lse=lse)
    if entropy is not None:
        out["entropy"] = entropy
    if top_ids is not None:
        out.update(top_ids=top_ids, top_logprobs=top_logprobs, rest=rest)
    return out


def _blocks(s):
    """(sequence, first, last + 1) in blocks of rows that the plain forms take at a time."""
    step = max(1, _CHUNK // s["case"]["V"])
    for b, t0, t1 in s["rows"]:
        for a in range(t0, t1, step):
            yield b, a, min(t1, a + step)


def _top(z, K):
    """The K largest of each row, equal ones in the order of their index."""
    V = z.shape[1]
    bits = (z + 0.0).view(torch.int32).long()
    order = torch.where(bits >= 0, bits, -(bits & 0x7fffffff))
    key = order * (1 << 28) + (V - 1 - torch.arange(V, device=z.device))
    return key.topk(K, dim=1).indices


def _plain_logprobs(s):
    c = s["case"]
    B, T, K = c["B"], c["T"], c["K"]
    dev = s["logits"].device
    logprob, lse, entropy = (torch.zeros((B, T), device=dev) for _ in range(3))
    ids = torch.full((B, T, K), -1, dtype=torch.int32, device=dev)
    top, rest = torch.zeros((B, T, K), device=dev), torch.zeros((B, T), device=dev)
    for b, t0, t1 in _blocks(s):
        z = s["logits"][b, t0:t1].float()
        m = z.max(dim=1, keepdim=True).values
        e = torch.exp(z - m)
        total = e.sum(dim=1, keepdim=True)
        norm = m + torch.log(total)
        lse[b, t0:t1] = norm[:, 0]
        logprob[b, t0:t1] = (z.gather(1, s["tokens"][b, t0:t1, None].long()) - norm)[:, 0]
        if c["entropy"]:
            entropy[b, t0:t1] = torch.log(total[:, 0]) + torch.where(e > 0, e * (m - z), 0.0).sum(dim=1) / total[:, 0]
        if K:
            j = _top(z, K)
            ids[b, t0:t1] = j.int()
            top[b, t0:t1] = z.gather(1, j) - norm
            rest[b, t0:t1] = torch.log(e.scatter(1, j, 0.0).sum(dim=1) / total[:, 0])
    return _scores(logprob, entropy if c["entropy"] else None, lse, ids if K else None, top, rest)


def _plain_grad(s):
    c = s["case"]
    for b, t0, t1 in _blocks(s):
        z = s["logits"][b, t0:t1].float()
        lp = z - s["lse"][b, t0:t1, None]
        p = torch.exp(lp)
        w = s["d_logprob"][b, t0:t1, None]
        g = -w * p
        if c["entropy"]:
            h = s["d_entropy"][b, t0:t1, None]
            g = g - torch.where(p > 0, h * p * (lp + s["entropy"][b, t0:t1, None]), 0.0)
        if c["K"]:
            d = s["d_top"][b, t0:t1]
            g = g - d.sum(dim=1, keepdim=True) * p
            g.scatter_add_(1, s["top_ids"][b, t0:t1].long(), d)
        g.scatter_add_(1, s["tokens"][b, t0:t1, None].long(), w)
        s["grad"][b, t0:t1] = g.to(s["grad"].dtype)
    return dict(grad=s["grad"])


def _rest_of(s, b, t0, t1):
    """Log of the teacher's mass outside its list."""
    if s["case"]["rest"]:
        return s["rest"][b, t0:t1]
    left = 1.0 - s["top_logprobs"][b, t0:t1].double().exp().sum(dim=1)
    return left.clamp(min=REST_FLOOR).log().float()


def _plain_topk_kl(s):
    c = s["case"]
    B, T = c["B"], c["T"]
    kl, logratio, gsq, lse = (torch.zeros((B, T), device=s["logits"].device) for _ in range(4))
    for b, t0, t1 in _blocks(s):
        z = s["logits"][b, t0:t1].float()
        m = z.max(dim=1, keepdim=True).values
        e = torch.exp(z - m)
        total = e.sum(dim=1, keepdim=True)
        norm = m + torch.log(total)
        j = s["top_ids"][b, t0:t1].long()
        p = e / total
        outside = torch.ones_like(p, dtype=torch.bool).scatter_(1, j, False)
        pr = torch.where(outside, p, 0.0).sum(dim=1, keepdim=True)
        lp, lq = z.gather(1, j) - norm, s["top_logprobs"][b, t0:t1]
        lpr, lqr = torch.log(pr), _rest_of(s, b, t0, t1)[:, None]
        d, dr = lp - lq, lpr - lqr
        if c["mode"] == "reverse":
            pj = torch.exp(lp)
            val = torch.where(pj > 0, pj * d, 0.0).sum(dim=1, keepdim=True) + pr * dr
            g = (p * (dr - val)).scatter_(1, j, torch.where(pj > 0, pj * (d - val), 0.0))
        else:
            val = -(torch.exp(lq) * d).sum(dim=1, keepdim=True) - torch.exp(lqr) * dr
            g = (p * (1.0 - torch.exp(-dr))).scatter_(1, j, torch.exp(lp) - torch.exp(lq))
        kl[b, t0:t1], lse[b, t0:t1] = val[:, 0], norm[:, 0]
        hit = j == s["tokens"][b, t0:t1, None].long()
        logratio[b, t0:t1] = torch.where(hit.any(dim=1), torch.where(hit, d, 0.0).sum(dim=1), dr[:, 0])
        gsq[b, t0:t1] = (g * g).sum(dim=1)
        s["grad"][b, t0:t1] = g.to(s["grad"].dtype)
    return dict(kl=kl, logratio=logratio, gsq=gsq, lse=lse, grad=s["grad"])


def _quantize(x):
    """Whole numbers in [-127, 127] and the step of each row: step = max|x| / 127, q = x / step rounded
    to nearest, ties to even, both in fp32."""
    x = x.float()
    step = x.abs().amax(dim=1) / torch.full((1,), 127.0, device=x.device)
    q = torch.where(step[:, None] > 0, torch.round(x / step[:, None]), 0.0)
    return q, step


def _plain_linear(s):
    q, step = _quantize(s["hidden"])
    q = q.double()                       # (sums of products pass 2^24)
    for v0 in range(0, s["case"]["V"], 16384):
        w = s["wq"][v0:v0 + 16384]
        acc = (q @ w.double().T).float()
        s["logits"][:, v0:v0 + 16384] = (acc * (step[:, None] * s["w_scale"][v0:v0 + 16384])).to(s["logits"].dtype)
    return dict(logits=s["logits"], scale=step)


_PLAIN = dict(logprobs=_plain_logprobs, logprobs_grad=_plain_grad, topk_kl=_plain_topk_kl,
              linear_i8=_plain_linear)
_OWN = dict(logprobs=_own_logprobs, logprobs_grad=_own_grad, topk_kl=_own_topk_kl,
            linear_i8=_own_linear)


# ----------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """What ``run`` returns for these inputs, in 64 bits from the definitions."""
    s = prepare(case, seed)
    if case["path"] == "linear_i8":
        return _exact_linear(s)
    out = {}
    ends = _ends(case)
    if case["path"] == "logprobs":
        names = ["logprob", "lse"] + (["entropy"] if case["entropy"] else [])
        out = {n: torch.zeros((case["B"], case["T"]), dtype=torch.float64, device="cuda") for n in names}
        if case["K"]:
            shape = (case["B"], case["T"], case["K"])
            out.update(top_ids=torch.full(shape, -1, dtype=torch.int32, device="cuda"),
                       top_logprobs=torch.zeros(shape, dtype=torch.float64, device="cuda"),
                       rest=torch.zeros(shape[:2], dtype=torch.float64, device="cuda"))
    elif case["path"] == "logprobs_grad":
        out = dict(grad=torch.zeros(tuple(s["grad"].shape), dtype=torch.float64, device="cuda"))
    else:
        out = {n: torch.zeros((case["B"], case["T"]), dtype=torch.float64, device="cuda")
               for n in ("kl", "logratio", "gsq", "lse")}
        out["grad"] = torch.zeros(tuple(s["grad"].shape), dtype=torch.float64, device="cuda")
    step = max(1, (_CHUNK // 2) // case["V"])
    for b in range(case["B"]):
        for t0 in range(0, ends[b], step):
            at = (b, slice(t0, min(ends[b], t0 + step)))
            for name, value in _EXACT[case["path"]](s, at).items():
                out[name][at] = value
    return out


def _probabilities(z):
    """Log-sum-exp, log probabilities and probabilities of each row."""
    z = z.double()
    lse = torch.logsumexp(z, dim=-1)
    lp = z - lse[..., None]
    return lse, lp, torch.exp(lp)


def _times(p, x):
    """p * x with 0 * inf = 0."""
    return torch.where(p == 0, torch.zeros((), dtype=p.dtype, device=p.device), p * x)


def _exact_logprobs(s, at):
    c, z = s["case"], s["logits"][at]
    lse, lp, p = _probabilities(z)
    out = dict(lse=lse, logprob=torch.take_along_dim(lp, s["tokens"][at][:, None].long(), 1)[:, 0])
    if c["entropy"]:
        out["entropy"] = -_times(p, lp).sum(dim=1)
    if c["K"]:
        order = torch.sort(z.float() + 0.0, dim=1, descending=True, stable=True).indices
        first = order[:, :c["K"]]
        out.update(top_ids=first.int(), top_logprobs=torch.take_along_dim(lp, first, 1),
                   rest=torch.take_along_dim(p, order[:, c["K"]:], 1).sum(dim=1).log())
    return out


def _exact_grad(s, at):
    # the definition takes the forward pass's log-sum-exp and entropy as they were given
    c, z = s["case"], s["logits"][at].double()
    lp = z - s["lse"][at].double()[:, None]
    p = torch.exp(lp)
    n, V = z.shape
    onto = torch.zeros_like(z)           # weight of each entry's own log probability
    onto[torch.arange(n, device="cuda"), s["tokens"][at].long()] = s["d_logprob"][at].double()
    if c["K"]:
        row = torch.arange(n, device="cuda")[:, None].expand(n, c["K"])
        onto.index_put_((row, s["top_ids"][at].long()), s["d_top"][at].double(), accumulate=True)
    grad = onto - p * onto.sum(dim=1, keepdim=True)
    if c["entropy"]:
        grad -= s["d_entropy"][at].double()[:, None] * _times(p, lp + s["entropy"][at].double()[:, None])
    return dict(grad=grad)


def _exact_topk_kl(s, at):
    c = s["case"]
    lse, lp, p = _probabilities(s["logits"][at])
    ids, lq = s["top_ids"][at].long(), s["top_logprobs"][at].double()
    n, K = ids.shape
    # categories: 0..K-1 the alternatives, K everything else
    cat = torch.full(lp.shape, K, dtype=torch.int64, device="cuda")
    cat[torch.arange(n, device="cuda")[:, None], ids] = torch.arange(K, device="cuda").expand(n, K)
    P = torch.zeros((n, K + 1), dtype=torch.float64, device="cuda")
    P[:, :K] = torch.take_along_dim(p, ids, 1)
    P[:, K] = torch.where(cat == K, p, 0.0).sum(dim=1)
    logP = torch.log(P)
    logP[:, :K] = torch.take_along_dim(lp, ids, 1)
    if c["rest"]:
        lr = s["rest"][at].double()
    else:
        lr = torch.log(torch.clamp(1.0 - torch.exp(lq).sum(dim=1), min=REST_FLOOR))
    logQ = torch.cat([lq, lr[:, None]], dim=1)
    D = logP - logQ
    if c["mode"] == "reverse":
        kl = _times(P, D).sum(dim=1)
        grad = _times(p, torch.take_along_dim(D, cat, 1) - kl[:, None])
    else:
        kl = -_times(torch.exp(logQ), D).sum(dim=1)
        grad = _times(p, 1.0 - torch.exp(-torch.take_along_dim(D, cat, 1)))
        top = torch.exp(logP[:, :K]) - torch.exp(lq)
        grad[torch.arange(n, device="cuda")[:, None], ids] = top
    mine = torch.take_along_dim(cat, s["tokens"][at][:, None].long(), 1)
    return dict(kl=kl, logratio=torch.take_along_dim(D, mine, 1)[:, 0], lse=lse, grad=grad,
                gsq=(grad * grad).sum(dim=1))


def _exact_linear(s):
    import numpy as np
    x = s["hidden"].float().cpu().numpy()
    step = np.abs(x).max(axis=1) / np.float32(127)          # (the definition rounds in fp32)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(step[:, None] > 0, np.rint(x / step[:, None]), np.float32(0))
    q = torch.from_numpy(q).cuda().double()
    out = torch.zeros(tuple(s["logits"].shape), dtype=torch.float64, device="cuda")
    scale = torch.from_numpy(step).cuda().double()
    for v0 in range(0, s["case"]["V"], 8192):
        w, sw = s["wq"][v0:v0 + 8192].double(), s["w_scale"][v0:v0 + 8192].double()
        out[:, v0:v0 + 8192] = torch.einsum("md,vd->mv", q, w) * scale[:, None] * sw[None, :]
    return dict(logits=out, scale=scale)


_EXACT = dict(logprobs=_exact_logprobs, logprobs_grad=_exact_grad, topk_kl=_exact_topk_kl)
