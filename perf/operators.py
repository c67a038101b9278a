"""Cases and plain forms of the attention-sublayer operators: rotary positions on the fused qkv array,
attention with modified scores (tanh cap, distance bias, document / prefix / window masks) forward and
backward, and counter-based dropout.

`own` False computes an operator with elementary torch operations in 32 bits (64 where an angle or a
position needs them); `own` True makes the calls of the package's binding.  Sizes are those of the
configurations in seeded_inputs.py (d_model 64, 768, 1024; 12 or 16 heads; 1,024 to 16,384 positions)
and odd ones between them.

Arrays follow include/bt.h: fused qkv [B*T, 3C] (columns q | k | v, head h at columns h*d .. of each
part).  Attention reads it the way the QKV projection leaves it: head_dim 64 and 128 as two FP32 planes
[2][B*T][3C] whose sum is the value, head_dim 16 and 32 as one raw array.
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda"


def listed():
    return [
        # one token far into a context: the latency of a single rotation
        rope("rope one token", "rope_fwd", B=1, T=1, C=768, H=12, far=100000),
        # one layer of the 124M model at batch 8, packed documents: positions restart inside a sequence
        rope("rope 124M", "rope_fwd", B=8, T=1024, C=768, H=12, mean=300),
        # gradient of a long-context layer: half of each head rotated, neighbouring pairs, frequencies
        # interpolated by wavelength beyond a trained length of 4,096
        rope("rope grad 16k", "rope_bwd", B=2, T=16381, C=1024, H=16, rot=32, inter=True, scaling=2, factor=8.0,
             low=1.0, high=4.0, length=4096, mscale=1.2),
        # one token's residual row
        dropout("dropout one row", "dropout_fwd", n=768, p=0.1, res=True),
        # residual branch of the 124M model at batch 8
        dropout("dropout 124M", "dropout_fwd", n=8192 * 768, p=0.1, res=True),
        # gradient of a 32,768 x 1,024 activation cut short of a multiple of four
        dropout("dropout grad", "dropout_bwd", n=32768 * 1024 - 1, p=0.25),
        # the tiny configuration's heads on short documents, padding at the end
        attention("attention tiny", "attn_fwd", B=2, T=65, C=64, H=4, mean=20, pad=9, slope=True),
        # one layer of the 124M model at batch 8: packed documents and a distance bias
        attention("attention 124M", "attn_fwd", B=8, T=1024, C=768, H=12, mean=400, slope=True),
        # 128-wide heads, a bidirectional prefix in front of each document, capped scores
        attention("attention wide prefix", "attn_fwd", B=2, T=1000, C=2048, H=16, mean=600, prefix=150, cap=30.0),
        # gradients: one layer of the 124M model, packed documents and capped scores
        attention("attention grad 124M", "attn_bwd", B=8, T=1024, C=768, H=12, mean=400, cap=30.0),
        # gradients: odd length, 32-wide heads, prefixes, distance bias, look-back window
        attention("attention grad narrow", "attn_bwd", B=3, T=777, C=256, H=8, mean=250, prefix=60, slope=True, window=200),
        # gradients of one long sequence: two or three documents with capped scores
        attention("attention grad 8k", "attn_bwd", B=1, T=8192, C=768, H=12, mean=4000, cap=50.0),
    ]


def rope(name, op, B, T, C, H, rot=0, inter=False, base=10000.0, scaling=0, factor=1.0, low=1.0, high=32.0, length=0,
         mscale=1.0, far=0, mean=0):
    return dict(name=name, op=op, B=B, T=T, C=C, H=H, rot=rot or C // H, inter=inter, base=base, scaling=scaling,
                factor=factor, low=low, high=high, length=length, mscale=mscale, far=far, mean=mean)


def dropout(name, op, n, p, res=False):
    return dict(name=name, op=op, n=n, p=p, res=res)


def attention(name, op, B, T, C, H, mean=0, pad=0, prefix=0, window=0, cap=0.0, slope=False, layout=1):
    return dict(name=name, op=op, B=B, T=T, C=C, H=H, mean=mean, pad=pad, prefix=prefix, window=window, cap=cap,
                slope=slope, layout=layout)


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("rope_fwd", "rope_bwd", "dropout_fwd", "dropout_bwd", "attn_fwd", "attn_fwd", "attn_bwd", "attn_bwd"))
    if op.startswith("dropout"):
        return unnamed(dropout("", op, n=log(1, 32768 * 1024 - 2), p=rng.choice((0.05, 0.1, 0.2, 0.5)),
                               res=op == "dropout_fwd" and rng.random() < 0.7))
    d = rng.choice((16, 32, 64, 64, 64, 128))
    H = rng.randint(1, 1536 // d)
    if op.startswith("rope"):
        B = rng.randint(1, 8)
        T = log(1, max(1, min(16384, 2 * 16381 * 1024 // (B * H * d) - 1)))
        return unnamed(rope("", op, B=B, T=T, C=H * d, H=H, rot=rng.choice((d, d, d // 2, d // 4 + d // 4 % 2)),
                            inter=rng.random() < 0.5, base=rng.choice((10000.0, 500000.0)), scaling=rng.randint(0, 2),
                            factor=rng.choice((2.0, 4.0, 8.0)), low=1.0, high=rng.choice((4.0, 32.0)),
                            length=rng.choice((1024, 2048, 4096)), mscale=rng.choice((1.0, 1.2)),
                            far=rng.choice((0, 0, 1000, 131072)), mean=rng.choice((0, 100, 1000))))
    B = rng.randint(1, 8)
    # no more score entries, and no more products, than the long listed case
    longest = int(math.sqrt(8192 * 8192 * 12 * min(1.0, 64 / d) / (B * H)))
    T = log(1, max(1, min(8191, longest)))
    return unnamed(attention("", op, B=B, T=T, C=H * d, H=H, mean=rng.choice((0, T // 8 + 1, T // 3 + 1)),
                             pad=rng.choice((0, 0, T // 10)), prefix=rng.choice((0, 0, T // 20 + 1, T // 5 + 1)),
                             window=rng.choice((0, 0, 0, T // 4 + 1)), cap=rng.choice((0.0, 0.0, 30.0, 50.0)),
                             slope=rng.random() < 0.4, layout=rng.randint(1, 1000)))


def unnamed(case):
    del case["name"]
    return case


# ------------------------------------------------------------------------------- inputs

def documents(case):
    """Document ids, prefix marks (both int32 [B, T]) and positions inside the documents of a packed batch.
    An id below zero marks padding.  The layout belongs to the case: work() counts its pairs."""
    B, T, mean = case["B"], case["T"], case["mean"]
    rng = random.Random(case.get("layout", 1))
    doc, mark = np.full((B, T), -1, np.int32), np.zeros((B, T), np.int32)
    pos = np.zeros((B, T), np.int32)
    for b in range(B):
        t, n, end = 0, 0, T - case.get("pad", 0)
        while t < end:
            size = min(end - t, rng.randint(1, 2 * mean) if mean else T)
            front = min(size, rng.randint(0, 2 * case["prefix"])) if case.get("prefix") else 0
            doc[b, t:t + size], mark[b, t:t + front], pos[b, t:t + size] = n, 1, np.arange(size)
            t, n = t + size, n + 1
    return doc, mark, pos


def slopes(H):
    """Geometric slopes 2^(-8 (h + 1) / H)."""
    return [2.0 ** (-8.0 * (h + 1) / H) for h in range(H)]


def prepare(case, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=DEVICE)  # noqa: E731
    state = {"case": case}
    if case["op"].startswith("dropout"):
        state["x"] = normal(case["n"])
        state["residual"] = normal(case["n"]) if case["res"] else None
        state["seed"], state["offset"] = seed * 2654435761 % (1 << 63), 3
        return state
    B, T, C, H = case["B"], case["T"], case["C"], case["H"]
    doc, mark, pos = documents(case)
    if case["op"].startswith("rope"):
        state["x"] = normal(B * T, 3 * C)
        state["pos"] = torch.from_numpy(pos.reshape(-1)).to(DEVICE) + case["far"]
        return state
    qkv, planes = normal(B * T, 3 * C), C // H >= 64
    state["qkv"] = split(qkv) if planes else qkv
    whole = not case["mean"] and not case["pad"] and not case["prefix"] and not case["window"]
    state["doc"] = None if whole else torch.from_numpy(doc).to(DEVICE)
    state["mark"] = torch.from_numpy(mark).to(DEVICE) if case["prefix"] else None
    state["slopes"] = torch.tensor(slopes(H), device=DEVICE) if case["slope"] else None
    if case["op"] == "attn_bwd":
        d_o = normal(B * T, C)
        state["o"], state["lse"] = attention_forward(state)
        state["d_o"] = split(d_o) if planes else d_o
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
    return {"rope_fwd": lambda s: rotate(s, 1.0), "rope_bwd": lambda s: rotate(s, -1.0), "dropout_fwd": drop,
            "dropout_bwd": drop, "attn_fwd": attention_forward, "attn_bwd": attention_backward}[op](state)


# ---- plain forms

def frequencies(case):
    """Radians per position of each rotated pair, 64 bits."""
    i = torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEVICE)
    f = case["base"] ** (-2.0 * i / case["rot"])
    if case["scaling"] == 1:
        f = f / case["factor"]
    elif case["scaling"] == 2:
        turns = case["length"] * f / (2.0 * math.pi)
        keep = ((turns - case["low"]) / (case["high"] - case["low"])).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / case["factor"])
    return f


def rotate(state, sign):
    case, x = state["case"], state["x"]
    H, rot = case["H"], case["rot"]
    angle = sign * state["pos"].double()[:, None] * frequencies(case)
    cos = (torch.cos(angle) * case["mscale"]).float()[:, None, None, :]
    sin = (torch.sin(angle) * case["mscale"]).float()[:, None, None, :]
    y = x.clone().view(x.shape[0], 3, H, -1)
    part = y[:, :2, :, :rot]
    if case["inter"]:
        a, b = part[..., 0::2].clone(), part[..., 1::2].clone()
        part[..., 0::2], part[..., 1::2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = part[..., :rot // 2].clone(), part[..., rot // 2:].clone()
        part[..., :rot // 2], part[..., rot // 2:] = a * cos - b * sin, a * sin + b * cos
    return y.view(x.shape)


def philox(blocks, seed, offset):
    """Four 32-bit words for each counter (block low, block high, offset low, offset high) and key `seed`:
    Philox-4x32 of ten rounds (Salmon, Moraes, Dror, Shaw 2011), [blocks, 4] as int64."""
    low = 0xFFFFFFFF
    i = torch.arange(blocks, device=DEVICE, dtype=torch.int64)
    c0, c1 = i & low, i >> 32
    c2, c3 = torch.full_like(i, offset & low), torch.full_like(i, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for r in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack((c0, c1, c2, c3), 1)


def drop(state):
    case, x = state["case"], state["x"]
    n, p = case["n"], case["p"]
    keep = philox((n + 3) // 4, state["seed"], state["offset"]).view(-1)[:n] >= round(p * 4294967296.0)
    y = torch.where(keep, x * (1.0 / (1.0 - p)), torch.zeros_like(x))
    return y if state["residual"] is None else y + state["residual"]


def visible(state):
    """[B, 1, T, T] truth values: may query i read key j."""
    case, doc = state["case"], state["doc"]
    T = case["T"]
    i = torch.arange(T, device=DEVICE)
    if doc is None:
        return (i[None, :] <= i[:, None])[None, None]
    new = torch.ones_like(doc, dtype=torch.bool)
    new[:, 1:] = doc[:, 1:] != doc[:, :-1]
    start = torch.where(new, i, torch.zeros_like(i)).cummax(1).values
    ok = (start[:, :, None] == start[:, None, :]) & (doc >= 0)[:, :, None]
    reach = i[None, None, :] <= i[None, :, None]
    if state["mark"] is not None:
        last = torch.where(state["mark"] == 0, i, torch.full_like(i, -1)).cummax(1).values
        reach = reach | (last < start)[:, None, :]
    if case["window"]:
        reach = reach & (i[:, None] - i[None, :] < case["window"])
    return (ok & reach)[:, None]


def heads(state):
    case = state["case"]
    B, T, H = case["B"], case["T"], case["H"]
    return value(state["qkv"]).view(B, T, 3, H, -1).permute(2, 0, 3, 1, 4)


def scores(state, q, k):
    """Modified scores before the mask, and tanh of the capped ones."""
    case = state["case"]
    s, t = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(q.shape[-1])), None
    if case["cap"]:
        t = torch.tanh(s / case["cap"])
        s = t * case["cap"]
    if state["slopes"] is not None:
        i = torch.arange(case["T"], device=DEVICE)
        s = s - state["slopes"][None, :, None, None] * (i[:, None] - i[None, :]).abs()
    return s, t


def attention_forward(state):
    case = state["case"]
    q, k, v = heads(state)
    s, _ = scores(state, q, k)
    s = torch.where(visible(state), s, torch.full_like(s, -math.inf))
    m = s.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(s - m)
    l = p.sum(3, keepdim=True)  # noqa: E741
    o = torch.matmul(p, v) / torch.where(l == 0, torch.ones_like(l), l)
    return o.permute(0, 2, 1, 3).reshape(-1, case["C"]), (m + torch.log(l))[..., 0]


def attention_backward(state):
    case = state["case"]
    B, T, C, H = case["B"], case["T"], case["C"], case["H"]
    q, k, v = heads(state)
    d_o = value(state["d_o"]).view(B, T, H, -1).permute(0, 2, 1, 3)
    dot = (d_o * state["o"].view(B, T, H, -1).permute(0, 2, 1, 3)).sum(3, keepdim=True)
    s, t = scores(state, q, k)
    p = torch.where(visible(state), torch.exp(s - state["lse"][..., None]), torch.zeros_like(s))
    dv = torch.matmul(p.transpose(2, 3), d_o)
    ds = p * (torch.matmul(d_o, v.transpose(2, 3)) - dot) * (1.0 / math.sqrt(q.shape[-1]))
    if t is not None:
        ds = ds * (1.0 - t * t)
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)
    return torch.stack((dq, dk, dv)).permute(1, 3, 0, 2, 4).reshape(B * T, 3 * C)


# ---- the framework's calls

def kept(state, make):
    """Output buffers and scratch, made at the first call as a program makes them once."""
    if "kept" not in state:
        state["kept"] = make()
    return state["kept"]


def empty(*shape):
    return torch.empty(*shape, device=DEVICE)


def own_rope(state, call):
    from paper_2606_24780_b200 import binding as b
    c, x = state["case"], state["x"]
    y, cfg = kept(state, lambda: (torch.empty_like(x), b.make_rope(
        c["rot"], c["inter"], c["base"], c["scaling"], c["factor"], c["low"], c["high"], c["length"], c["mscale"])))
    getattr(b, call)(x, state["pos"], c["B"] * c["T"], c["T"], c["C"], c["H"], cfg, y)
    return y


def own_dropout_fwd(state):
    from paper_2606_24780_b200 import binding as b
    c, x = state["case"], state["x"]
    y = kept(state, lambda: torch.empty_like(x))
    b.bt_op_dropout_fwd(x, state["residual"], c["n"], c["p"], state["seed"], state["offset"], y)
    return y


def own_dropout_bwd(state):
    from paper_2606_24780_b200 import binding as b
    c, x = state["case"], state["x"]
    dx = kept(state, lambda: torch.empty_like(x))
    b.bt_op_dropout_bwd(x, c["n"], c["p"], state["seed"], state["offset"], dx)
    return dx


def own_mod(state, b):
    """The score modification of this batch; the key spans are built from the document ids in every pass."""
    c = state["case"]
    B, T = c["B"], c["T"]
    if "mod" not in state:
        state["spans"] = None
        if state["doc"] is not None:
            state["spans"] = torch.empty(b.bt_op_attention_spans_bytes(B, T), dtype=torch.uint8, device=DEVICE)
        state["mod"] = b.make_attn_mod(c["cap"], state["slopes"], state["spans"])
        state["scratch"] = torch.empty(b.bt_op_attention_mod_scratch_bytes(B, T, c["C"], c["H"]), dtype=torch.uint8,
                                       device=DEVICE)
    if state["spans"] is not None:
        b.bt_op_attention_spans(state["doc"], state["mark"], c["window"], B, T, state["spans"], state["spans"].numel())
    return state["mod"], state["scratch"]


def raw_or_planes(x):
    return (None, x) if x.dim() == 3 else (x, None)


def own_attention_fwd(state):
    from paper_2606_24780_b200 import binding as b
    c = state["case"]
    B, T, C, H = c["B"], c["T"], c["C"], c["H"]
    mod, scratch = own_mod(state, b)
    o, lse = kept(state, lambda: (empty(B * T, C), empty(B, H, T)))
    b.bt_op_attention_mod_fwd(*raw_or_planes(state["qkv"]), B, T, C, H, mod, o, None, lse, scratch,
                              scratch.numel())
    return o, lse


def own_attention_bwd(state):
    from paper_2606_24780_b200 import binding as b
    c = state["case"]
    B, T, C, H = c["B"], c["T"], c["C"], c["H"]
    mod, scratch = own_mod(state, b)
    dqkv = kept(state, lambda: empty(B * T, 3 * C))
    b.bt_op_attention_mod_bwd(*raw_or_planes(state["qkv"]), state["o"], state["lse"], *raw_or_planes(state["d_o"]),
                              B, T, C, H, mod, dqkv, None, scratch, scratch.numel())
    return dqkv


OWN = {"rope_fwd": lambda s: own_rope(s, "bt_op_rope_fwd"), "rope_bwd": lambda s: own_rope(s, "bt_op_rope_bwd"),
       "dropout_fwd": own_dropout_fwd, "dropout_bwd": own_dropout_bwd, "attn_fwd": own_attention_fwd,
       "attn_bwd": own_attention_bwd}


# ------------------------------------------------------------------------------- bytes and operations

def pairs(case):
    """(query, key) pairs one head of the whole batch scores."""
    doc, mark, pos = documents(case)
    total = 0
    for row, marks in zip(doc, mark):
        cuts = np.flatnonzero(np.diff(row)) + 1
        for ids, front in zip(np.split(row, cuts), np.split(marks, cuts)):
            if ids[0] >= 0:
                i = np.arange(len(ids))
                low = np.maximum(0, i - case["window"] + 1) if case["window"] else 0
                total += int(np.sum(np.maximum(i + 1, int(front.sum())) - low))
    return total


def work(case):
    if case["op"].startswith("dropout"):
        return {"bytes": (12 if case["res"] else 8) * case["n"], "flops": 3 * case["n"]}
    n, C, H = case["B"] * case["T"], case["C"], case["H"]
    if case["op"].startswith("rope"):
        return {"bytes": 24 * n * C + 4 * n, "flops": 6 * n * H * case["rot"]}
    products = 2 * pairs(case) * C
    if case["op"] == "attn_fwd":
        return {"bytes": n * (12 * C + 4 * C + 4 * H), "flops": 2 * products}
    return {"bytes": n * (12 * C + 8 * C + 4 * H + 12 * C), "flops": 5 * products}


# ------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    state = prepare(case, seed)
    if case["op"].startswith("dropout"):
        return exact_dropout(state)
    if case["op"].startswith("rope"):
        return exact_rope(state)
    return exact_attention(state)


def exact_rope(state):
    """Each pair as a complex number times mscale e^(i angle)."""
    c, x = state["case"], state["x"].double()
    H, rot = c["H"], c["rot"]
    freq = []
    for i in range(rot // 2):
        f = math.exp(-2.0 * i / rot * math.log(c["base"]))
        if c["scaling"] == 1:
            f /= c["factor"]
        if c["scaling"] == 2:
            keep = min(1.0, max(0.0, (c["length"] / (2.0 * math.pi / f) - c["low"]) / (c["high"] - c["low"])))
            f = keep * f + (1.0 - keep) * f / c["factor"]
        freq.append(f if c["op"] == "rope_fwd" else -f)
    angle = torch.outer(state["pos"].double(), torch.tensor(freq, dtype=torch.float64, device=DEVICE))
    turn = torch.polar(torch.full_like(angle, c["mscale"]), angle)[:, None, None, :]
    y = x.view(x.shape[0], 3, H, -1).clone()
    part = y[:, :2, :, :rot]
    if c["inter"]:
        z = torch.view_as_complex(part.unflatten(3, (-1, 2)).contiguous()) * turn
        y[:, :2, :, :rot] = torch.view_as_real(z).flatten(3)
    else:
        z = torch.complex(*part.chunk(2, 3)) * turn
        y[:, :2, :, :rot] = torch.cat((z.real, z.imag), 3)
    return y.view(x.shape)


def exact_dropout(state):
    """The same generator with its 32 x 32-bit products built from 16-bit halves."""
    c, seed, offset = state["case"], state["seed"], state["offset"]

    def product(a, m):
        ah, al, mh, ml = a // 65536, a % 65536, m // 65536, m % 65536
        low = al * ml
        mid = ah * ml + low // 65536
        mid2 = al * mh + mid % 65536
        return ah * mh + mid // 65536 + mid2 // 65536, (mid2 % 65536) * 65536 + low % 65536

    i = torch.arange((c["n"] + 3) // 4, device=DEVICE, dtype=torch.int64)
    word = [i % 2 ** 32, i // 2 ** 32, torch.full_like(i, offset % 2 ** 32), torch.full_like(i, offset // 2 ** 32)]
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for _ in range(10):
        (h0, l0), (h1, l1) = product(word[0], 0xD2511F53), product(word[2], 0xCD9E8D57)
        word = [h1 ^ word[1] ^ key[0], l1, h0 ^ word[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    kept_values = torch.stack(word, 1).reshape(-1)[:c["n"]].double() >= round(c["p"] * 2.0 ** 32)
    y = state["x"].double() / (1.0 - c["p"]) * kept_values
    return y if state["residual"] is None else y + state["residual"].double()


def exact_attention(state):
    """softmax over the visible keys of each row, one head at a time; gradients by automatic differentiation."""
    c = state["case"]
    B, T, C, H = c["B"], c["T"], c["C"], c["H"]
    d, back = C // H, c["op"] == "attn_bwd"
    doc, mark, _ = documents(c)
    x = value(state["qkv"].double()).view(B, T, 3, H, d)
    o = torch.zeros(B, T, H, d, dtype=torch.float64, device=DEVICE)
    lse = torch.full((B, H, T), -math.inf, dtype=torch.float64, device=DEVICE)
    grad = torch.zeros(B, T, 3, H, d, dtype=torch.float64, device=DEVICE)
    for b in range(B):
        edges = [0] + [int(t) for t in np.flatnonzero(np.diff(doc[b])) + 1] + [T]
        for s, e in zip(edges[:-1], edges[1:]):
            if doc[b, s] < 0:
                continue
            i = torch.arange(e - s, device=DEVICE)
            front = int(mark[b, s:e].sum())
            see = (i[None, :] <= i[:, None]) | (i[None, :] < front)
            if c["window"]:
                see &= i[:, None] - i[None, :] < c["window"]
            step = max(1, min(H, (1 << 27) // max(1, (e - s) ** 2)))
            for h in range(0, H, step):
                part = x[b, s:e, :, h:h + step].permute(1, 2, 0, 3).clone().requires_grad_(back)
                z = part[0] @ part[1].transpose(1, 2) / math.sqrt(d)
                if c["cap"]:
                    z = c["cap"] * torch.tanh(z / c["cap"])
                if c["slope"]:
                    z = z - state["slopes"][h:h + step, None, None].double() * (i[:, None] - i[None, :]).abs()
                z = z.masked_fill(~see, -math.inf)
                out = torch.softmax(z, 2) @ part[2]
                o[b, s:e, h:h + step] = out.detach().permute(1, 0, 2)
                lse[b, h:h + step, s:e] = torch.logsumexp(z.detach(), 2)
                if back:
                    g = value(state["d_o"].double()).view(B, T, H, d)[b, s:e, h:h + step].permute(1, 0, 2)
                    out.backward(g)
                    grad[b, s:e, :, h:h + step] = part.grad.permute(2, 0, 1, 3)
    return grad.view(B * T, 3 * C) if back else (o.view(B * T, C), lse)
