"""The operators over the vocabulary, as they are measured: log probabilities of given tokens with entropy and
top alternatives (remoe_token_logprobs), their gradient (remoe_token_logprobs_backward), distillation from a
teacher's top logits (remoe_distill_forward) and its gradient (remoe_distill_backward).

With z [T, V] the logits, tau the temperature, m the largest logit of a row and d = (z - m) / tau:

  S = sum_v exp(d_v) = 1 + rest,  p_v = exp(d_v) / S,  stats = (m, rest)
  logprob = ln p_target,  entropy = ln S - sum_v d_v exp(d_v) / S,  alternatives: the largest z, ties to the lower id
  dlogits_v = (1/tau) (g_l (1[v = target] - p_v) - g_H p_v (ln p_v + entropy))
  q = softmax(t / tau) over the teacher's K listed logits t, or exp(t / tau - lse) with the teacher's own normaliser
  loss = sum_j q_j (ln q_j - ln p_id(j)),  dlogits_v = (g / tau) (p_v sum_j q_j - sum_{j: id_j = v} q_j)

`run` computes them from elementary torch operations, or calls the library where `own` is true.  Logits are
Gaussian around an uneven popularity of the tokens, with the given token well above the rest; the teacher's are the
student's with noise.  Padded rows are views of wider buffers.
"""
import math

import torch

own = False

DEV = "cuda:0"
TOKENS = 8192              # the ranges that `draw` covers
VOCAB = (1000, 152000)
ELEMENTS = TOKENS * 151936


def _case(name, kind, tokens, vocab, dtype, tau=1.0, top=0, entropy=False, k=0, lse=False, masked=False, pad=0):
    return {"name": name, "kind": kind, "tokens": tokens, "vocab": vocab, "dtype": dtype, "tau": tau, "top": top,
            "entropy": entropy, "k": k, "lse": lse, "masked": masked, "pad": pad}


def listed():
    return [
        # one token of one request: log probabilities and twenty alternatives, latency counts
        _case("logprobs_one_token", "logprobs", 1, 151936, "bf16", 0.7, top=20, entropy=True),
        # a step of 64 requests under a grammar's mask, five alternatives each
        _case("logprobs_batch64_masked", "logprobs", 64, 102400, "bf16", 1.0, top=5, entropy=True, masked=True),
        # a prompt of odd length scored in full precision, an odd vocabulary: no row but the first is aligned
        _case("logprobs_prompt1021_f32", "logprobs", 1021, 50257, "f32", entropy=True),
        # a teacher's top 64 taken for a later distillation
        _case("logprobs_top64", "logprobs", 2048, 32000, "bf16", top=64),
        # the forward pass of a training step of 4 sequences of 2048 tokens
        _case("logprobs_train8k", "logprobs", 8192, 151936, "bf16", entropy=True),
        # the gradient for a few sampled tokens
        _case("logprobs_grad_batch16_f32", "logprobs_grad", 16, 32000, "f32", 0.7),
        # policy gradient with an entropy bonus on a ragged batch, odd vocabulary
        _case("logprobs_grad_1021", "logprobs_grad", 1021, 50257, "bf16", 1.0, entropy=True),
        # the backward pass of the training step
        _case("logprobs_grad_train8k", "logprobs_grad", 8192, 151936, "bf16"),
        # distillation on one ragged prompt, the teacher's normaliser kept with its logits
        _case("distill_prompt333", "distill", 333, 102400, "bf16", 2.0, k=64, lse=True),
        # a training step's distillation, logits in a buffer padded to a multiple of 128
        _case("distill_train4k", "distill", 4096, 151936, "bf16", 1.0, k=128),
        # the gradients of both
        _case("distill_grad_prompt333_f32", "distill_grad", 333, 102400, "f32", 2.0, k=64, lse=True),
        _case("distill_grad_train4k", "distill_grad", 4096, 151936, "bf16", 1.0, k=128, pad=64),
    ]


def draw(rng):
    def log_uniform(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))

    kind = rng.choice(["logprobs", "logprobs_grad", "distill", "distill_grad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    vocab = log_uniform(*VOCAB)
    if rng.random() < 0.5:
        vocab = max(VOCAB[0], vocab // 8 * 8)
    most = ELEMENTS // (1 if dtype == "bf16" else 2) // vocab
    tokens = min(log_uniform(1, TOKENS), most)
    teacher = kind.startswith("distill")
    return {"kind": kind, "tokens": tokens, "vocab": vocab, "dtype": dtype, "tau": rng.choice([0.6, 0.7, 1.0, 1.0, 2.0, 4.0]),
            "top": rng.choice([0, 1, 5, 20, 64]) if kind == "logprobs" else 0,
            "entropy": not teacher and rng.random() < 0.5, "k": log_uniform(1, 256) if teacher else 0,
            "lse": teacher and rng.random() < 0.5, "masked": rng.random() < 0.25,
            "pad": rng.choice([0, 0, 0, rng.randrange(1, 129)])}


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _teacher(case):
    return case["kind"].startswith("distill")


def _blocks(case, elements=1 << 26):
    """Ranges of rows of at most so many logits: what is made or checked in pieces."""
    rows = max(1, elements // case["vocab"])
    return [(r, min(r + rows, case["tokens"])) for r in range(0, case["tokens"], rows)]


def prepare(case, seed):
    T, V, tau = case["tokens"], case["vocab"], case["tau"]
    g = torch.Generator(device=DEV).manual_seed(seed)
    buf = torch.empty(T, V + case["pad"], dtype=_dtype(case), device=DEV)
    z = buf[:, :V]
    targets = torch.randint(0, V, (T,), generator=g, device=DEV)
    popularity = -torch.log1p(torch.randperm(V, generator=g, device=DEV).float())     # a token's rank, Zipf's law
    if case["pad"]:
        buf[:, V:] = float("nan")                                                      # never read
    for a, b in _blocks(case):
        block = torch.randn(b - a, V, generator=g, device=DEV).mul_(2.0).add_(popularity)
        if case["masked"]:
            block.masked_fill_(torch.rand(b - a, V, generator=g, device=DEV) < 0.9, -math.inf)
        row = torch.arange(b - a, device=DEV)
        block[row, targets[a:b]] = 4.0 + 4.0 * torch.rand(b - a, generator=g, device=DEV)
        z[a:b] = block
    state = {"case": case, "logits": z, "targets": targets.int()}

    if _teacher(case):
        K = case["k"]
        ids = torch.empty(T, K, dtype=torch.int64, device=DEV)
        tl = torch.empty(T, K, device=DEV)
        for a, b in _blocks(case):
            zb = z[a:b].float()
            vals, at = torch.topk(zb, K, dim=1)
            ids[a:b] = at
            vals = torch.where(vals > -math.inf, vals, torch.full_like(vals, -12.0))
            tl[a:b] = vals + torch.randn(b - a, K, generator=g, device=DEV)
        # what the list leaves of the teacher's distribution: between nothing and a fifth
        state["teacher_idx"] = ids.int()
        state["teacher_logits"] = tl
        state["teacher_lse"] = None
        if case["lse"]:
            rest = 1.0 - 0.2 * torch.rand(T, generator=g, device=DEV)
            state["teacher_lse"] = torch.logsumexp(tl / tau, 1) - torch.log(rest)

    if case["kind"] == "logprobs":
        n = case["top"]
        state["out"] = {"logprob": torch.empty(T, device=DEV), "stats": torch.empty(T, 2, device=DEV)}
        if case["entropy"]:
            state["out"]["entropy"] = torch.empty(T, device=DEV)
        if n:
            state["out"]["top_idx"] = torch.empty(T, n, dtype=torch.int32, device=DEV)
            state["out"]["top_logprob"] = torch.empty(T, n, device=DEV)
    elif case["kind"] == "distill":
        state["out"] = {"loss": torch.empty(T, device=DEV), "stats": torch.empty(T, 2, device=DEV)}
    else:
        # what the forward pass has left behind, and the gradient that comes from above
        stats, entropy = torch.empty(T, 2, device=DEV), torch.empty(T, device=DEV)
        for a, b in _blocks(case):
            m, rest, d, e = _row_sums(z[a:b], tau)
            stats[a:b, 0], stats[a:b, 1] = m, rest
            entropy[a:b] = torch.log1p(rest) - torch.where(e > 0, d * e, 0.0).sum(1) / (1.0 + rest)
        state["stats"] = stats
        state["d_row"] = (0.5 + torch.rand(T, generator=g, device=DEV)) / T * (1.0 if _teacher(case) else -1.0)
        state["entropy"] = state["d_entropy"] = None
        if case["entropy"]:
            state["entropy"] = entropy
            state["d_entropy"] = 0.1 * torch.randn(T, generator=g, device=DEV) / T
        grad = torch.empty(T, V + case["pad"], dtype=_dtype(case), device=DEV)
        state["out"] = {"dlogits": grad[:, :V]}

    if own:
        import paper_2605_27081_amd as remoe

        state["desc"] = remoe.HeadDesc(V, remoe.REMOE_BF16 if case["dtype"] == "bf16" else remoe.REMOE_F32, tau)
        if case["kind"] in ("logprobs", "distill"):
            size = remoe.remoe_head_workspace_bytes(state["desc"], T, case["top"])
            state["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    return state


# ---- the plain form ---------------------------------------------------------------------------

def _row_sums(z, tau):
    """Largest logit, the sum of all exponentials but its own (which is 1), differences, exponentials."""
    z = z.float()
    m, at = z.max(1, keepdim=True)
    d = (z - m) / tau
    e = torch.exp(d)
    return m[:, 0], e.scatter(1, at, 0.0).sum(1), d, e


def _alternatives(z, n):
    """Ids of the n largest logits, ties to the lower id: the logits as integers of the same order above the ids."""
    bits = (z.float() + 0.0).view(torch.int32).long()
    order = torch.where(bits >= 0, bits, -2147483648 - bits)
    keys = order * (1 << 31) - torch.arange(z.shape[1], device=z.device)
    return (-torch.topk(keys, n, dim=1).values) % (1 << 31)


def _plain_logprobs(s):
    case, z = s["case"], s["logits"]
    m, rest, d, e = _row_sums(z, case["tau"])
    log_s = torch.log1p(rest)
    out = {"logprob": d.gather(1, s["targets"].long()[:, None])[:, 0] - log_s, "stats": torch.stack([m, rest], 1)}
    if case["entropy"]:
        out["entropy"] = log_s - torch.where(e > 0, d * e, 0.0).sum(1) / (1.0 + rest)
    if case["top"]:
        ids = _alternatives(z, case["top"])
        out["top_idx"] = ids.int()
        out["top_logprob"] = d.gather(1, ids) - log_s[:, None]
    return out


def _plain_logprobs_grad(s):
    case, z, tau = s["case"], s["logits"], s["case"]["tau"]
    m, rest, at = s["stats"][:, :1], s["stats"][:, 1:], s["targets"].long()[:, None]
    d = (z.float() - m) / tau
    p = torch.exp(d) / (1.0 + rest)
    g = -s["d_row"][:, None] * p
    # 1 - p cancels where the target has nearly everything: in 64 bits from the rest of the sum
    short = rest.double() - torch.expm1((z.gather(1, at).double() - m.double()) / tau)
    g.scatter_(1, at, (s["d_row"].double()[:, None] * short / (1.0 + rest.double())).float())
    if s["d_entropy"] is not None:
        log_p = d - torch.log1p(rest)
        g -= s["d_entropy"][:, None] * torch.where(p > 0, p * (log_p + s["entropy"][:, None]), 0.0)
    return {"dlogits": (g / tau).to(z.dtype)}


def _plain_teacher(s):
    """q and ln q of the listed tokens: few, and differences of them count, so in 64 bits."""
    t = s["teacher_logits"].double() / s["case"]["tau"]
    lse = None if s["teacher_lse"] is None else s["teacher_lse"].double()
    if lse is None:
        top = t.amax(1)
        lse = top + torch.log(torch.exp(t - top[:, None]).sum(1))
    log_q = t - lse[:, None]
    return torch.exp(log_q), log_q


def _plain_distill(s):
    case, z = s["case"], s["logits"]
    m, rest, d, _ = _row_sums(z, case["tau"])
    q, log_q = _plain_teacher(s)
    log_p = d.gather(1, s["teacher_idx"].long()).double() - torch.log1p(rest.double())[:, None]
    return {"loss": (q * (log_q - log_p)).sum(1).float(), "stats": torch.stack([m, rest], 1)}


def _plain_distill_grad(s):
    z, tau, at = s["logits"], s["case"]["tau"], s["teacher_idx"].long()
    m, rest = s["stats"][:, :1], s["stats"][:, 1:]
    q, _ = _plain_teacher(s)
    mass = q.sum(1, keepdim=True)
    g = torch.exp((z.float() - m) / tau) * (mass / (1.0 + rest.double())).float()
    # where the teacher has a share the difference cancels: (e M - q (1 + rest)) / S in 64 bits
    less = torch.expm1((z.gather(1, at).double() - m.double()) / tau)
    g.scatter_(1, at, ((less * mass + (mass - q) - q * rest.double()) / (1.0 + rest.double())).float())
    return {"dlogits": (g * (s["d_row"][:, None] / tau)).to(z.dtype)}


PLAIN = {"logprobs": _plain_logprobs, "logprobs_grad": _plain_logprobs_grad,
         "distill": _plain_distill, "distill_grad": _plain_distill_grad}


def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        return PLAIN[kind](s)
    import paper_2605_27081_amd as remoe

    out = s["out"]
    if kind == "logprobs":
        remoe.remoe_token_logprobs(s["desc"], s["logits"], s["targets"], out["logprob"], out.get("entropy"), out.get("top_idx"),
                                   out.get("top_logprob"), out["stats"], s["workspace"])
    elif kind == "logprobs_grad":
        remoe.remoe_token_logprobs_backward(s["desc"], s["logits"], s["stats"], s["targets"], s["d_row"], s["entropy"],
                                            s["d_entropy"], out["dlogits"])
    elif kind == "distill":
        remoe.remoe_distill_forward(s["desc"], s["logits"], s["teacher_idx"], s["teacher_logits"], s["teacher_lse"], out["loss"],
                                    out["stats"], s["workspace"])
    else:
        remoe.remoe_distill_backward(s["desc"], s["logits"], s["stats"], s["teacher_idx"], s["teacher_logits"], s["teacher_lse"],
                                     s["d_row"], out["dlogits"])
    return out


def work(case):
    T, V, n, k = case["tokens"], case["vocab"], case["top"], case["k"]
    logits = T * V * (2 if case["dtype"] == "bf16" else 4)
    teacher = T * (8 * k + (4 if case["lse"] else 0))
    # an element's difference, scaling, exponential, sum and comparison; the entropy's product and sum
    flops = T * V * (5 + (2 if case["entropy"] else 0))
    if case["kind"] == "logprobs":
        return {"bytes": logits + T * (4 + 4 + 8 + (4 if case["entropy"] else 0) + 8 * n), "flops": flops}
    if case["kind"] == "logprobs_grad":
        return {"bytes": 2 * logits + T * (8 + 4 + 4 + (8 if case["entropy"] else 0)), "flops": flops}
    if case["kind"] == "distill":
        return {"bytes": logits + teacher + T * (4 + 8), "flops": flops + 8 * T * k}
    return {"bytes": 2 * logits + teacher + T * (8 + 4), "flops": flops + 4 * T * k}


# ---- the definitions in 64 bits ----------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    tau, parts = case["tau"], []
    for a, b in _blocks(case, 1 << 25):
        x = s["logits"][a:b].double() / tau
        log_p = torch.log_softmax(x, 1)
        if _teacher(case):
            ids = s["teacher_idx"][a:b].long()
            t = s["teacher_logits"][a:b].double() / tau
            log_q = torch.log_softmax(t, 1) if s["teacher_lse"] is None else t - s["teacher_lse"][a:b].double()[:, None]
            q = log_q.exp()
        out = {}
        if case["kind"] in ("logprobs", "distill"):
            top = x.max(1, keepdim=True).values
            out["stats"] = torch.cat([top * tau, torch.expm1(torch.logsumexp(x - top, 1, keepdim=True))], 1)
        if case["kind"] == "logprobs":
            rows = torch.arange(b - a, device=DEV)
            out["logprob"] = log_p[rows, s["targets"][a:b].long()]
            if case["entropy"]:
                out["entropy"] = torch.special.entr(log_p.exp()).sum(1)
            if case["top"]:
                ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
                out["top_idx"], out["top_logprob"] = ids.int(), torch.gather(log_p, 1, ids)
        elif case["kind"] == "distill":
            out["loss"] = (q * (log_q - log_p.gather(1, ids))).sum(1)
        else:
            # from the statistics in hand, as the gradient's definition has them
            p = torch.exp(x - s["stats"][a:b, :1].double() / tau) / (1.0 + s["stats"][a:b, 1:].double())
            up = s["d_row"][a:b].double()[:, None]
            if case["kind"] == "logprobs_grad":
                one = torch.zeros_like(p).scatter_(1, s["targets"][a:b].long()[:, None], 1.0)
                grad = up * (one - p)
                if s["d_entropy"] is not None:
                    ln_p = torch.log(p)
                    inner = torch.where(p > 0, p * (ln_p + s["entropy"][a:b].double()[:, None]), 0.0)
                    grad = grad - s["d_entropy"][a:b].double()[:, None] * inner
            else:
                grad = up * (p * q.sum(1, keepdim=True) - torch.zeros_like(p).scatter_add_(1, ids, q))
            out["dlogits"] = grad / tau
        parts.append(out)
    # in the order in which run() names them
    names = {"logprobs": ["logprob", "stats", "entropy", "top_idx", "top_logprob"], "distill": ["loss", "stats"]}.get(case["kind"], ["dlogits"])
    return {n: torch.cat([p[n] for p in parts]) for n in names if n in parts[0]}
