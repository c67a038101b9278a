"""Cases and plain forms of the losses at the language-model head: softmax cross entropy from hidden states
without keeping the logits, distillation from a teacher's top logits in the same form, each forward and
backward, and distillation on logits at hand.

`own` False computes an operator with elementary torch operations in 32 bits; `own` True makes the calls of
the package's binding.  Sizes are those of the configurations in seeded_inputs.py (d_model 64, 768, 1024;
vocabularies of 512, 50,257 and 50,304; 1 to 8,192 rows) and odd ones between them.

Arrays follow include/bt.h: hidden states x [N, C], head weights w [V, C], row-major FP32, raw or as the two
planes [2][rows][C] whose sum is the value, the form in which the training step keeps both.
"""
import math

import torch

own = False

DEVICE = "cuda"


def listed():
    return [
        # the log-probability of one token: latency, one read of the weights
        head("xent one token", "xent_fwd", N=1, C=768, V=50257),
        # one short document scored at d_model 1,024
        head("xent short document", "xent_fwd", N=100, C=1024, V=50257),
        # loss of the 124M model at batch 8, operands as the training step keeps them
        head("xent 124M", "xent_fwd", N=8192, C=768, V=50304, planes=True),
        # gradients from a handful of rows (the answer tokens of one short example)
        head("xent grad few rows", "xent_bwd", N=5, C=1024, V=50257, pad=0.2),
        # gradients of the 124M model's head at batch 8
        head("xent grad 124M", "xent_bwd", N=8192, C=768, V=50304, planes=True),
        # gradients with row weights and padding rows, odd rows and vocabulary
        head("xent grad ragged", "xent_bwd", N=1999, C=512, V=32001, weights=True, pad=0.1),
        # the tiny configuration's student
        head("distill tiny", "distill_fwd", N=256, C=64, V=512, K=8, tau=1.0),
        # two sequences of a 124M student against a teacher's 64 best logits
        head("distill 124M", "distill_fwd", N=2048, C=768, V=50304, K=64, tau=2.0, planes=True),
        # gradients at d_model 1,024; the teacher's probabilities are those of its whole vocabulary
        head("distill grad 1024", "distill_bwd", N=4096, C=1024, V=50304, K=32, tau=1.5, whole=True, planes=True, pad=0.05),
        # logits at hand: one row
        logits("distill logits one row", N=1, V=50304, K=16, tau=2.0),
        # logits of the 124M model at batch 8, padded columns behind the vocabulary
        logits("distill logits 124M", N=8192, V=50257, K=64, tau=2.0),
        # a vocabulary of 2^17 - 1, rows without a teacher's entry among them
        logits("distill logits wide", N=513, V=131071, K=100, tau=1.0, whole=True, pad=0.1),
    ]


def head(name, op, N, C, V, K=0, tau=1.0, whole=False, weights=False, pad=0.0, planes=False):
    return dict(name=name, op=op, N=N, C=C, V=V, K=K, tau=tau, whole=whole, weights=weights, pad=pad, planes=planes)


def logits(name, N, V, K, tau, whole=False, weights=False, pad=0.0):
    return head(name, "logits", N, 0, V, K, tau, whole, weights, pad)


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("xent_fwd", "xent_fwd", "xent_bwd", "xent_bwd", "distill_fwd", "distill_bwd", "logits", "logits"))
    K = 0 if op.startswith("xent") else log(1, 128)
    V = max(K, log(500, 131000))
    tau = rng.choice((1.0, 1.5, 2.0, 4.0)) if K else 1.0
    more = dict(K=K, tau=tau, whole=K > 0 and rng.random() < 0.3, weights=rng.random() < 0.3, pad=rng.choice((0.0, 0.0, 0.05, 0.3)))
    if op == "logits":
        case = head("", op, N=log(1, max(1, min(8191, 8192 * 50257 // V - 1))), C=0, V=V, **more)
    else:
        C = 32 * log(2, 48)
        case = head("", op, N=log(1, max(1, min(8191, 8192 * 50304 * 768 // (V * C) - 1))), C=C, V=V,
                    planes=rng.random() < 0.5, **more)
    del case["name"]
    return case


# ------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=DEVICE)  # noqa: E731
    uniform = lambda n: torch.rand(n, generator=gen, device=DEVICE)  # noqa: E731
    N, C, V, K = case["N"], case["C"], case["V"], case["K"]
    state = {"case": case, "inv": 1.0 / N}
    empty_row = uniform(N) < case["pad"]
    if case["pad"] and N > 1:
        empty_row[0], empty_row[1] = True, False
    state["row_w"] = 2.0 * uniform(N) if case["weights"] else None
    if case["op"] == "logits":
        ld = (V + 63) // 64 * 64
        state["logits"] = 3.0 * normal(N, ld)
    else:
        x, w = normal(N, C), normal(V, C) * (3.0 / math.sqrt(C))
        state["x"], state["w"] = (split(x), split(w)) if case["planes"] else (x, w)
    if K:
        # distinct ids: an arithmetic walk that is shorter than the vocabulary
        first, step = (uniform(N) * V).long().clamp(max=V - 1), 1 + (uniform(N) * (V // K - 1)).long()
        ids = (first[:, None] + step[:, None] * torch.arange(K, device=DEVICE)) % V
        top = (4.0 + 3.0 * normal(N, K)).sort(1, descending=True).values
        ids[empty_row] = -1
        if K > 2 and N > 2:
            ids[2::3, K - 1] = -1                                     # a row with fewer entries
        state["ids"], state["top"] = ids.int(), top
        state["top_lse"] = None
        if case["whole"]:                                             # the rest of the teacher's vocabulary holds a tenth
            state["top_lse"] = (top.double() / case["tau"]).logsumexp(1).float() + 0.1
    else:
        target = (uniform(N) * V).long().clamp(max=V - 1)
        target[empty_row] = -1
        state["target"] = target.int()
    if case["op"].endswith("_bwd"):
        state["lse"] = row_lse(scores(state))
    return state


def split(x):
    """The two planes of bt.h: the value rounded to ten mantissa bits, and the rest."""
    hi = ((x.view(torch.int32) + 0x1000) & ~0x1FFF).view(torch.float32)
    return torch.stack((hi, x - hi))


def value(x):
    return x[0] + x[1] if x.dim() == 3 else x


# ------------------------------------------------------------------------------- one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return OWN[op](state)
    return {"xent_fwd": head_forward, "distill_fwd": head_forward, "xent_bwd": head_backward, "distill_bwd": head_backward,
            "logits": logits_pass}[op](state)


# ---- plain forms

def scores(state):
    return torch.matmul(value(state["x"]), value(state["w"]).t()) * (1.0 / state["case"]["tau"])


def row_lse(z):
    m = z.amax(1)
    return m + torch.log(torch.exp(z - m[:, None]).sum(1))


def teacher(state):
    """Columns [N, K] and probabilities p [N, K] of the aim of each row; zeros in the place of absent entries."""
    if "target" in state:
        t = state["target"].long()[:, None]
        return t.clamp(min=0), (t >= 0).float()
    ids, tau = state["ids"].long(), state["case"]["tau"]
    t = torch.where(ids >= 0, state["top"] * (1.0 / tau), torch.full_like(state["top"], -math.inf))
    if state["top_lse"] is not None:
        return ids.clamp(min=0), torch.exp(t - state["top_lse"][:, None])
    m = t.amax(1, keepdim=True)
    e = torch.exp(t - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = e.sum(1, keepdim=True)
    return ids.clamp(min=0), e / torch.where(total == 0, torch.ones_like(total), total)


def losses_of(state, z, lse):
    ids, p = teacher(state)
    log_p = torch.log(torch.where(p > 0, p, torch.ones_like(p)))
    losses = state["case"]["tau"] ** 2 * (p * (log_p + (lse[:, None] - z.gather(1, ids)))).sum(1)
    weighted = losses if state["row_w"] is None else losses * state["row_w"]
    return losses, (weighted.double().sum(0, keepdim=True) * state["inv"]).float()


def score_gradient(state, z, lse):
    ids, p = teacher(state)
    d = torch.exp(z - lse[:, None]) * p.sum(1, keepdim=True)
    d.scatter_add_(1, ids, -p)
    g = state["inv"] * state["case"]["tau"]
    return d * (g if state["row_w"] is None else g * state["row_w"][:, None])


def head_forward(state):
    z = scores(state)
    lse = row_lse(z)
    losses, mean = losses_of(state, z, lse)
    return {"losses": losses, "lse": lse, "mean": mean}


def head_backward(state):
    d = score_gradient(state, scores(state), state["lse"])
    return {"dx": torch.matmul(d, value(state["w"])), "dw": torch.matmul(d.t(), value(state["x"]))}


def logits_pass(state):
    V = state["case"]["V"]
    z = state["logits"][:, :V] * (1.0 / state["case"]["tau"])
    lse = row_lse(z)
    losses, mean = losses_of(state, z, lse)
    grad = torch.zeros_like(state["logits"])
    grad[:, :V] = score_gradient(state, z, lse)
    return {"losses": losses, "mean": mean, "grad": grad}


# ---- the framework's calls

def kept(state, make):
    """Output buffers and scratch, made at the first call as a program makes them once."""
    if "kept" not in state:
        state["kept"] = make()
    return state["kept"]


def empty(*shape):
    return torch.empty(*shape, device=DEVICE)


def scratch(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device=DEVICE)


def raw_or_planes(x):
    return (None, x) if x.dim() == 3 else (x, None)


def aim(state, b):
    """What the rows are held to: targets, or the teacher's entries."""
    if "target" in state:
        return state["target"]
    return b.make_distill(state["ids"], state["top"], state["case"]["tau"], state["top_lse"])


def own_head_fwd(state):
    from paper_2606_24780_b200 import binding as b
    c = state["case"]
    N, C, V, K = c["N"], c["C"], c["V"], c["K"]
    losses, lse, mean, work = kept(state, lambda: (empty(N), empty(N), empty(1), scratch(b.bt_op_head_fwd_scratch_bytes(N, C, V, K))))
    call = b.bt_op_head_distill_fwd if K else b.bt_op_head_xent_fwd
    call(*raw_or_planes(state["x"]), *raw_or_planes(state["w"]), aim(state, b), state["row_w"], N, C, V, state["inv"], losses,
         lse, mean, work, work.numel())
    return {"losses": losses, "lse": lse, "mean": mean}


def own_head_bwd(state):
    from paper_2606_24780_b200 import binding as b
    c = state["case"]
    N, C, V, K = c["N"], c["C"], c["V"], c["K"]
    dx, dw, work = kept(state, lambda: (empty(N, C), empty(V, C), scratch(b.bt_op_head_bwd_scratch_bytes(N, C, V, K))))
    call = b.bt_op_head_distill_bwd if K else b.bt_op_head_xent_bwd
    call(*raw_or_planes(state["x"]), *raw_or_planes(state["w"]), aim(state, b), state["row_w"], state["lse"], N, C, V,
         state["inv"], dx, dw, work, work.numel())
    return {"dx": dx, "dw": dw}


def own_logits(state):
    from paper_2606_24780_b200 import binding as b
    c, z = state["case"], state["logits"]
    losses, mean, grad = kept(state, lambda: (empty(c["N"]), empty(1), torch.empty_like(z)))
    b.bt_op_softmax_distill(z, aim(state, b), state["row_w"], c["N"], c["V"], z.shape[1], state["inv"], losses, mean, grad)
    return {"losses": losses, "mean": mean, "grad": grad}


OWN = {"xent_fwd": own_head_fwd, "distill_fwd": own_head_fwd, "xent_bwd": own_head_bwd, "distill_bwd": own_head_bwd,
       "logits": own_logits}


# ------------------------------------------------------------------------------- bytes and operations

def work(case):
    N, C, V, K = case["N"], case["C"], case["V"], case["K"]
    rows = N * (8 * K + 4 + (4 if case["weights"] else 0) + (4 if case["whole"] else 0) + (0 if K else 4))
    if case["op"] == "logits":
        return {"bytes": 8 * N * V + rows, "flops": 5 * N * V}
    if case["op"].endswith("_fwd"):
        return {"bytes": 4 * (N + V) * C + rows + 4 * N, "flops": 2 * N * V * C}
    return {"bytes": 8 * (N + V) * C + rows, "flops": 6 * N * V * C}


# ------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    """Row blocks with the aim of each row as a dense distribution."""
    s, c = prepare(case, seed), case
    N, V, K, tau, back = c["N"], c["V"], c["K"], c["tau"], c["op"].endswith("_bwd")
    x = w = None
    if c["op"] != "logits":
        x, w = (s[k].double().sum(0) if s[k].dim() == 3 else s[k].double() for k in ("x", "w"))
    f64 = dict(dtype=torch.float64, device=DEVICE)
    losses, lse = torch.zeros(N, **f64), torch.zeros(N, **f64)
    dx = dw = grad = None
    if back:
        dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    if c["op"] == "logits":
        grad = torch.zeros(s["logits"].shape, **f64)
    weight = torch.ones(N, **f64) if s["row_w"] is None else s["row_w"].double()
    block = max(1, (1 << 27) // V)
    for a in range(0, N, block):
        e = min(N, a + block)
        z = (s["logits"][a:e, :V].double() if x is None else x[a:e] @ w.T) / tau
        p, entropy = torch.zeros(e - a, V + 1, **f64), torch.zeros(e - a, **f64)
        if K:
            ids = s["ids"][a:e].long()
            t = (s["top"][a:e].double() / tau).masked_fill(ids < 0, -math.inf)
            log_p = t - s["top_lse"][a:e, None].double() if c["whole"] else torch.log_softmax(t, 1)
            prob = torch.exp(log_p).nan_to_num(0.0)
            entropy = torch.special.entr(prob).sum(1)
            p.scatter_add_(1, torch.where(ids < 0, torch.full_like(ids, V), ids), prob)
        else:
            t = s["target"][a:e].long()
            p.scatter_(1, torch.where(t < 0, torch.full_like(t, V), t)[:, None], 1.0)
        p = p[:, :V]
        lse[a:e] = torch.logsumexp(z, 1)
        losses[a:e] = tau ** 2 * ((p * (lse[a:e, None] - z)).sum(1) - entropy)
        if back or grad is not None:
            norm = s["lse"][a:e].double() if back else lse[a:e]
            d = (torch.exp(z - norm[:, None]) * p.sum(1, keepdim=True) - p) * (weight[a:e, None] * tau * s["inv"])
            if back:
                dx[a:e] = d @ w
                dw += d.T @ x[a:e]
            else:
                grad[a:e, :V] = d
    if back:
        return {"dx": dx, "dw": dw}
    mean = (losses * weight).sum(0, keepdim=True) * s["inv"]
    if grad is not None:
        return {"losses": losses, "mean": mean, "grad": grad}
    return {"losses": losses, "lse": lse, "mean": mean}
