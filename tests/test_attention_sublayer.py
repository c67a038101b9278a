"""Rotary positions, key spans, attention with modified scores and dropout, against plain 64-bit forms.

Tolerances.  Half a rounding of an FP32 value is 2^-24 of it; the products of the tensor-core kernels
are sums of three TF32 products (dropped part: 2^-22 of a product) in an accumulator that truncates (2^-23
of the running sum per instruction, 24 instructions for 64 columns, so at most 24 * 2^-23 = 3e-6 of a score and
half of that on average).  A score error e moves a probability by e, so with scores of a few units an output
or gradient is within 1e-5 of its norm; the plain FP32 kernels are well inside that.
"""
import math
import threading

import numpy as np
import pytest
import torch

from paper_2606_24780_b200 import binding as b
from paper_2606_24780_b200 import build as bt_build

from gpu_util import DEV, check_split, rel_l2

gpu = pytest.mark.gpu
TOL = 1e-5


# ------------------------------------------------------------------------------- 64-bit forms

def see_matrix(doc, prefix, window, B, T):
    """[B, T, T] truth values, straight from the definition of the spans."""
    see = np.zeros((B, T, T), bool)
    for n in range(B):
        ids = [0] * T if doc is None else [int(v) for v in doc[n]]
        marks = [0] * T if prefix is None else [int(v) for v in prefix[n]]
        s = 0
        while s < T:
            e = s
            while e < T and ids[e] == ids[s]:
                e += 1
            p = s
            while p < e and marks[p] != 0:
                p += 1
            if ids[s] >= 0:
                for i in range(s, e):
                    for j in range(s, e):
                        see[n, i, j] = (j <= i or j < p) and (window == 0 or i - j < window)
            s = e
    return see


def attention64(qkv, see, cap, slopes, d_o=None):
    """qkv [B, T, 3, H, d], d_o [B, T, H, d] (64-bit, any device) -> o, lse and, with d_o, dqkv."""
    q, k, v = qkv.permute(2, 0, 3, 1, 4)
    d, T = q.shape[-1], q.shape[2]
    s = q @ k.transpose(2, 3) / math.sqrt(d)
    t = torch.tanh(s / cap) if cap else torch.zeros_like(s)
    z = cap * t if cap else s
    i = torch.arange(T, device=s.device)
    if slopes is not None:
        z = z - slopes[None, :, None, None] * (i[:, None] - i[None, :]).abs()
    z = z.masked_fill(~see[:, None], -math.inf)
    lse = torch.logsumexp(z, 3)
    p = torch.where(see[:, None], torch.exp(z - torch.where(lse == -math.inf, 0.0, lse)[..., None]), 0.0)
    o = p @ v
    if d_o is None:
        return o.permute(0, 2, 1, 3), lse
    g = d_o.permute(0, 2, 1, 3)
    ds = p * (g @ v.transpose(2, 3) - (g * o).sum(3, keepdim=True)) * (1 - t * t) / math.sqrt(d)
    grad = torch.stack((ds @ k, ds.transpose(2, 3) @ q, p.transpose(2, 3) @ g), 0)    # [3, B, H, T, d]
    # Before it cancels: do_i v_j and do_i o_i are each rounded on their own, so their difference is known to an
    # error relative to the two, not to itself (where a row reads one key it is zero, and so are dq and dk).
    # The norms of dq and dk with the two added as independent errors would be:
    w = p ** 2 * ((g @ v.transpose(2, 3)) ** 2 + (g * o).sum(3, keepdim=True) ** 2) * (1 - t * t) ** 2 / d
    size = [float((w @ k ** 2).sum().sqrt()), float((w.transpose(2, 3) @ q ** 2).sum().sqrt()), 0.0]
    return o.permute(0, 2, 1, 3), lse, grad.permute(1, 3, 0, 2, 4), size


def rope64(x, pos, H, rot, inter, theta, mscale, sign=1.0):
    """x [N, 3C] (numpy, 64-bit)."""
    y = x.reshape(x.shape[0], 3, H, -1).copy()
    for i in range(rot // 2):
        u, w = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        a = sign * np.asarray(pos, np.float64) * theta[i]
        c, s = (np.cos(a) * mscale)[:, None, None], (np.sin(a) * mscale)[:, None, None]
        pu, pw = y[:, :2, :, u].copy(), y[:, :2, :, w].copy()
        y[:, :2, :, u], y[:, :2, :, w] = pu * c - pw * s, pu * s + pw * c
    return y.reshape(x.shape)


def thetas(rot, base=10000.0, scaling=0, factor=1.0, low=1.0, high=32.0, length=0):
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if scaling == 1:
            f /= factor
        if scaling == 2:
            keep = min(1.0, max(0.0, (length * f / (2 * math.pi) - low) / (high - low)))
            f *= keep + (1 - keep) / factor
        out.append(f)
    return out


def philox(counter, key):
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep_mask(n, p, seed, offset, first_block=0):
    out = []
    for blk in range(first_block, first_block + (n + 3) // 4):
        out += philox((blk & 0xFFFFFFFF, blk >> 32, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))
    return np.array(out[:n], np.uint64) >= round(p * 2 ** 32)


# ------------------------------------------------------------------------------- CPU: refusals, generator

@pytest.fixture(scope="module")
def lib():
    bt_build.build()
    return b.lib()


def test_generator_gives_the_published_words():
    assert philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    f = 0xFFFFFFFF
    assert philox((f, f, f, f), (f, f)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


A = 0x10000   # an aligned address that no refused call reads


def refused(status, call, *args, **kw):
    with pytest.raises(b.BtError) as e:
        call(*args, stream=0, **kw)
    assert e.value.status == status, e.value


def test_rope_refusals(lib):
    ok = b.make_rope(64)
    refused(1, b.bt_op_rope_fwd, None, None, 4, 4, 768, 12, ok, A)
    refused(1, b.bt_op_rope_fwd, A + 4, None, 4, 4, 768, 12, ok, A)
    refused(1, b.bt_op_rope_fwd, A, None, 4, 4, 768, 12, ok, None)
    refused(1, b.bt_op_rope_fwd, A, None, -1, 4, 768, 12, ok, A)
    refused(1, b.bt_op_rope_fwd, A, None, 4, 0, 768, 12, ok, A)
    refused(1, b.bt_op_rope_fwd, A, None, 4, 4, 768, 7, ok, A)
    refused(1, b.bt_op_rope_fwd, A, None, 4, 4, 18, 3, b.make_rope(6), A)           # head_dim 6
    refused(1, b.bt_op_rope_fwd, A, None, 4, 4, 768, 12, ok, A, y_split=A)          # planes over the input
    refused(1, b.bt_op_rope_bwd, A, None, 4, 4, 768, 12, ok, A, dx_split=A << 8)    # in place and planes
    for bad in (b.make_rope(0), b.make_rope(3), b.make_rope(66), b.make_rope(64, base=0.0), b.make_rope(64, base=math.inf),
                b.make_rope(64, scaling=3), b.make_rope(64, scaling=1, factor=0.5), b.make_rope(64, mscale=math.nan),
                b.make_rope(64, scaling=2, factor=2.0), b.make_rope(64, scaling=2, factor=2.0, original_len=10, low=4, high=4)):
        refused(1, b.bt_op_rope_fwd, A, None, 4, 4, 768, 12, bad, A)
    b.bt_op_rope_fwd(A, None, 0, 4, 768, 12, ok, A, stream=0)                        # nothing to do


def test_spans_refusals(lib):
    n = b.bt_op_attention_spans_bytes(2, 100)
    assert n >= 2 * 2 * 100 * 8
    assert b.bt_op_attention_spans_bytes(0, 4) == b.bt_op_attention_spans_bytes(4, 0) == 0
    assert b.bt_op_attention_spans_bytes(1, (1 << 21) + 1) == b.bt_op_attention_spans_bytes(1 << 12, 1 << 20) == 0
    refused(1, b.bt_op_attention_spans, A, None, 0, 2, 100, None, n)
    refused(1, b.bt_op_attention_spans, A + 4, None, 0, 2, 100, A, n)
    refused(1, b.bt_op_attention_spans, A, None, -1, 2, 100, A, n)
    refused(1, b.bt_op_attention_spans, A, None, 0, 0, 100, A, n)
    refused(2, b.bt_op_attention_spans, A, None, 0, 1, (1 << 21) + 1, A, 1 << 40)
    refused(3, b.bt_op_attention_spans, A, None, 0, 2, 100, A, n - 1)


def test_attention_mod_refusals(lib):
    mod = b.make_attn_mod()
    n = b.bt_op_attention_mod_scratch_bytes(2, 100, 128, 2)

    def fwd(status, qkv=A, split=None, B=2, T=100, C=128, H=2, mod=mod, o=A, o_split=None, lse=A, scratch=A, size=n):
        refused(status, b.bt_op_attention_mod_fwd, qkv, split, B, T, C, H, mod, o, o_split, lse, scratch, size)

    def bwd(status, o=A, lse=A, d_o=A, dqkv=A, scratch=A, size=n, H=2):
        refused(status, b.bt_op_attention_mod_bwd, A, None, o, lse, d_o, None, 2, 100, 128, H, mod, dqkv, None, scratch, size)

    fwd(1, qkv=None), fwd(1, qkv=A + 8), fwd(1, B=0), fwd(1, T=0), fwd(1, H=3), fwd(1, o=None), fwd(1, lse=None), fwd(1, scratch=None)
    fwd(1, scratch=A + 16), fwd(2, H=1, C=96), fwd(2, H=16), fwd(3, size=n - 1), fwd(2, T=(1 << 21) + 1, size=1 << 40)
    fwd(2, B=1 << 13, T=1 << 18, size=1 << 50)
    fwd(1, mod=b.make_attn_mod(softcap=-1.0)), fwd(1, mod=b.make_attn_mod(softcap=math.inf)), fwd(1, mod=b.make_attn_mod(softcap=math.nan))
    fwd(1, mod=b.make_attn_mod(slopes=A + 4)), fwd(1, mod=b.make_attn_mod(spans=A + 8))
    fwd(1, mod=b.make_attn_mod(softcap=1e-21)), fwd(1, mod=b.make_attn_mod(softcap=2e20)), fwd(1, qkv=A, o=A), fwd(1, o=None, o_split=A)
    bwd(1, dqkv=A), bwd(1, o=2 * A, dqkv=2 * A), bwd(1, d_o=3 * A, dqkv=3 * A)
    bwd(1, o=None), bwd(1, lse=None), bwd(1, d_o=None), bwd(1, dqkv=None), bwd(1, scratch=None), bwd(3, size=n - 1), bwd(1, H=3)
    refused(1, b.bt_op_attention_mod_check, None)
    # the C entries take a NULL modification
    assert lib.bt_op_attention_mod_fwd(A, None, 2, 100, 128, 2, None, A, None, A, A, n, 0, None) == 1
    assert lib.bt_op_rope_fwd(A, None, 2, 100, 128, 2, None, A, None, None) == 1


def test_dropout_refusals(lib):
    refused(1, b.bt_op_dropout_fwd, None, None, 8, 0.1, 1, 2, A)
    refused(1, b.bt_op_dropout_fwd, A, A + 4, 8, 0.1, 1, 2, A)
    refused(1, b.bt_op_dropout_fwd, A, None, 8, 0.1, 1, 2, None)
    refused(1, b.bt_op_dropout_fwd, A, None, -8, 0.1, 1, 2, A)
    refused(1, b.bt_op_dropout_fwd, A, None, 7, 0.1, 1, 2, None, y_split=A)
    refused(1, b.bt_op_dropout_fwd, A, None, 8, 0.1, 1, 2, A, d_step=A + 4)
    for p in (-0.1, 1.0, 1.5, math.nan):
        refused(1, b.bt_op_dropout_bwd, A, 8, p, 1, 2, A)
    b.bt_op_dropout_fwd(A, None, 0, 0.1, 1, 2, A, stream=0)


def test_tensors_of_another_type_or_place_are_refused(lib):
    cpu = torch.zeros(8)
    with pytest.raises(ValueError):
        b.bt_op_dropout_fwd(cpu, None, 8, 0.1, 1, 2, cpu, stream=0)
    with pytest.raises(ValueError):
        b.bt_op_dropout_fwd(cpu.double(), None, 8, 0.1, 1, 2, cpu, stream=0)
    with pytest.raises(ValueError):
        b.make_attn_mod(slopes=cpu)


# ------------------------------------------------------------------------------- rotary positions

def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV)


def np64(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


ROPE = [
    # N, H, d, rot, interleaved, positions, scaling arguments
    (1, 12, 64, 64, False, [100000], {}),
    (7, 3, 64, 64, True, [0, 1, 2, 2147483647, -5, 131072, 1048575], {}),
    (37, 2, 128, 128, False, None, dict(base=500000.0, scaling=2, factor=8.0, low=1.0, high=4.0, length=16)),
    (130, 5, 32, 16, True, None, dict(scaling=1, factor=4.0)),
    (33, 2, 16, 6, False, None, {}),                       # 3 pairs: the scalar form
    (33, 1, 16, 2, True, None, dict(mscale=1.3)),
    (1000, 12, 64, 32, False, None, dict(mscale=0.7)),
    (300, 1, 256, 128, True, None, {}),                    # a head wider than the rotated part
    (3, 1, 4, 4, False, None, {}),
]


@gpu
@pytest.mark.parametrize("N,H,d,rot,inter,pos,extra", ROPE)
def test_rope(N, H, d, rot, inter, pos, extra):
    C, T = H * d, max(1, N // 2)
    extra = dict(extra)
    mscale = extra.pop("mscale", 1.0)
    theta = thetas(rot, **extra)
    args = dict(extra)
    if "length" in args:
        args["original_len"] = args.pop("length")
    cfg = b.make_rope(rot, inter, mscale=mscale, **args)
    m = float(np.float32(mscale))
    x = rand(1, N, 3 * C)
    p = None if pos is None else torch.tensor(pos, dtype=torch.int32, device=DEV)
    at = np.arange(N) % T if pos is None else np.array(pos, np.int64)
    guard = torch.full((N + 2, 3 * C), 7.0, device=DEV)
    planes = torch.empty(2, N, 3 * C, device=DEV)
    for call, sign in ((b.bt_op_rope_fwd, 1.0), (b.bt_op_rope_bwd, -1.0)):
        y = guard[1:1 + N]
        call(x, p, N, T, C, H, cfg, y, planes)
        want = rope64(np64(x), at, H, rot, inter, theta, m, sign)
        # two products and a sum per value, sine and cosine within 2^-22, each of at most |u| + |w|
        pair = rope_magnitude(np64(x), H, rot, inter)
        assert (np.abs(np64(y) - want) <= 8 * 2.0 ** -24 * m * pair + 1e-30).all()
        assert (guard[0] == 7).all() and (guard[-1] == 7).all()
        check_split(planes, y.cpu().numpy())
        again = x.clone()
        call(again, p, N, T, C, H, cfg, again)
        assert torch.equal(again, y)
        only = torch.empty_like(planes)
        call(x, p, N, T, C, H, cfg, None, only)
        assert torch.equal(only, planes)
    # the columns that do not turn are copied bit for bit
    part = y.view(N, 3, H, d)
    assert torch.equal(part[:, 2], x.view(N, 3, H, d)[:, 2]) and torch.equal(part[..., rot:], x.view(N, 3, H, d)[..., rot:])


def rope_magnitude(x, H, rot, inter):
    y = np.abs(x.reshape(x.shape[0], 3, H, -1))
    out = y.copy()
    for i in range(rot // 2):
        u, w = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        out[:, :2, :, u] = out[:, :2, :, w] = y[:, :2, :, u] + y[:, :2, :, w]
    return out.reshape(x.shape)


@gpu
def test_rope_backward_undoes_a_pure_rotation():
    N, H, d = 200, 4, 64
    x, y, z = rand(2, N, 3 * H * d), torch.empty(N, 3 * H * d, device=DEV), torch.empty(N, 3 * H * d, device=DEV)
    cfg = b.make_rope(64)
    b.bt_op_rope_fwd(x, None, N, 50, H * d, H, cfg, y)
    b.bt_op_rope_bwd(y, None, N, 50, H * d, H, cfg, z)
    assert rel_l2(np64(z), np64(x)) < 8 * 2.0 ** -24


# ------------------------------------------------------------------------------- key spans

def spans_of(doc, prefix, window, B, T):
    buf = torch.empty(b.bt_op_attention_spans_bytes(B, T), dtype=torch.uint8, device=DEV)
    put = lambda a: None if a is None else torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)  # noqa: E731
    b.bt_op_attention_spans(put(doc), put(prefix), window, B, T, buf, buf.numel())
    return buf


def random_layout(rng, B, T, mean, pad, prefix):
    doc, mark = np.full((B, T), -1, np.int32), (rng.random((B, T)) < 0.3).astype(np.int32) if prefix else None
    for n in range(B):
        t, k, end = 0, int(rng.integers(0, 5)), T - (int(rng.integers(0, pad + 1)) if pad else 0)
        while t < end:
            size = min(end - t, int(rng.integers(1, 2 * mean + 1)))
            doc[n, t:t + size] = k if rng.random() < 0.9 or not pad else -int(rng.integers(1, 4))
            if prefix:
                mark[n, t:t + min(size, int(rng.integers(0, 2 * prefix + 1)))] = 1
            t, k = t + size, k + 1
    return doc, mark


@gpu
@pytest.mark.parametrize("B,T,mean,pad,prefix,window", [
    (1, 1, 1, 0, 0, 0), (2, 3, 1, 1, 1, 1), (3, 64, 20, 10, 5, 0), (2, 65, 30, 0, 8, 7), (2, 130, 200, 129, 60, 0),
    (1, 200, 9, 40, 3, 5), (2, 129, 40, 0, 0, 2147483647)])
def test_spans_follow_the_definition(B, T, mean, pad, prefix, window):
    doc, mark = random_layout(np.random.default_rng(B * 1000 + T), B, T, mean, pad, prefix)
    raw = spans_of(doc, mark, window, B, T).view(torch.int32).cpu().numpy().reshape(-1, 2)
    n, nb = B * T, (T + 63) // 64
    k, q, kb, qb = raw[:n], raw[n:2 * n], raw[2 * n:2 * n + B * nb], raw[2 * n + B * nb:]
    see = see_matrix(doc, mark, window, B, T)
    for s in range(B):
        for i in range(T):
            want = np.flatnonzero(see[s, i])
            lo, hi = k[s * T + i]
            assert list(want) == list(range(lo, hi))
            want = np.flatnonzero(see[s, :, i])
            lo, hi = q[s * T + i]
            assert list(want) == list(range(lo, hi))
        for blk in range(nb):
            for rows, got in ((see[s], kb), (see[s].T, qb)):
                cols = np.flatnonzero(rows[blk * 64:(blk + 1) * 64].any(0))
                lo, hi = got[s * nb + blk]
                assert (lo, hi) == ((cols[0], cols[-1] + 1) if len(cols) else (0, 0))


@gpu
def test_spans_of_long_sequences():
    """More than one chunk of the kernel's scans: documents that cross, start at and end at chunk edges."""
    T, rng = 20001, np.random.default_rng(5)
    doc = np.zeros((2, T), np.int32)
    doc[1] = np.repeat(np.arange(T // 5000 + 1), 5000)[:T]
    doc[1, 4090:4100] = -1
    mark = np.zeros((2, T), np.int32)
    mark[0, :4096] = 1
    mark[1, 10000:13000] = 1
    lone = np.zeros((2, T), np.int32)        # one document per sequence, all of the first and 9,000 of the second in the prefix
    lone[0], lone[1, :9000] = 1, 1
    for ids, marks in ((doc, mark), (None, lone), (np.zeros((2, T), np.int32), None)):
        check_long_spans(ids, marks, T, rng)


def check_long_spans(ids, marks, T, rng):
    doc, mark = np.zeros((2, T), np.int32) if ids is None else ids, np.zeros((2, T), np.int32) if marks is None else marks
    for window in (0, 300):
        raw = spans_of(ids, marks, window, 2, T).view(torch.int32).cpu().numpy().reshape(-1, 2)
        for s in range(2):
            cuts = [0] + list(np.flatnonzero(np.diff(doc[s])) + 1) + [T]
            for a, e in zip(cuts[:-1], cuts[1:]):
                p = a + (int(np.argmin(mark[s, a:e])) if (mark[s, a:e] == 0).any() else e - a)
                for i in {a, e - 1, min(e - 1, a + 1), (a + e) // 2, min(e - 1, p), max(a, p - 1), *rng.integers(a, e, 20)}:
                    lo, hi = raw[s * T + i]
                    qlo, qhi = raw[2 * T + s * T + i]
                    if doc[s, a] < 0:
                        assert lo >= hi and qlo >= qhi
                        continue
                    assert (lo, hi) == (max(a, i - window + 1) if window else a, max(i + 1, p))
                    assert (qlo, qhi) == (a if i < p else i, min(e, i + window) if window else e)


# ------------------------------------------------------------------------------- attention

def planes_of(x):
    out = torch.empty(2, *x.shape, device=DEV)
    b.bt_op_split(x, x.numel(), out) if x.numel() % 4 == 0 else out.copy_(torch.stack((x, torch.zeros_like(x))))
    return out


class Case:
    """One call's inputs and its 64-bit answer."""

    def __init__(self, B, T, H, d, cap=0.0, slope=False, mean=0, pad=0, prefix=0, window=0, seed=0, scale=1.0, doc=None, mark=None):
        self.B, self.T, self.H, self.d, self.C = B, T, H, d, H * d
        self.qkv = rand(seed + 1, B * T, 3 * self.C) * scale
        self.d_o = rand(seed + 2, B * T, self.C)
        self.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device=DEV) if slope else None
        self.spans = None
        see = np.broadcast_to(np.tril(np.ones((T, T), bool)), (B, T, T))
        if mean or pad or prefix or window or doc is not None:
            if doc is None:
                doc, mark = random_layout(np.random.default_rng(seed + 7 * T), B, T, mean or T, pad, prefix)
            see = see_matrix(doc, mark, window, B, T) if T < 400 else see_fast(doc, mark, window, B, T)
            self.spans = spans_of(doc, mark, window, B, T)
        self.mod = b.make_attn_mod(cap, self.slopes, self.spans)
        self.o, self.lse, self.grad, self.size = attention64(
            self.qkv.double().view(B, T, 3, H, d), torch.tensor(np.ascontiguousarray(see), device=DEV), cap,
            None if self.slopes is None else self.slopes.double(), self.d_o.double().view(B, T, H, d))
        size = b.bt_op_attention_mod_scratch_bytes(B, T, self.C, H)
        self.scratch = torch.full((size,), 255, dtype=torch.uint8, device=DEV)

    def forward(self, planes, flags=0, planes_out=False):
        B, T, C, H = self.B, self.T, self.C, self.H
        guard = torch.full((B * T + 2, C), 7.0, device=DEV)
        lse = torch.full((B * H * T + 8,), 7.0, device=DEV)
        o, split = guard[1:-1], torch.empty(2, B * T, C, device=DEV) if planes_out else None
        x = (None, planes_of(self.qkv)) if planes else (self.qkv, None)
        b.bt_op_attention_mod_fwd(*x, B, T, C, H, self.mod, o, split, lse, self.scratch, self.scratch.numel(), flags)
        b.bt_op_attention_mod_check(self.scratch)
        assert (guard[0] == 7).all() and (guard[-1] == 7).all() and (lse[B * H * T:] == 7).all()
        if planes_out:
            check_split(split, o.cpu().numpy())
        return o, lse[:B * H * T].view(B, H, T)

    def backward(self, planes, flags=0, planes_out=False):
        B, T, C, H = self.B, self.T, self.C, self.H
        guard = torch.full((B * T + 2, 3 * C), 7.0, device=DEV)
        dqkv, split = guard[1:-1], torch.empty(2, B * T, 3 * C, device=DEV) if planes_out else None
        x = (None, planes_of(self.qkv)) if planes else (self.qkv, None)
        g = (None, planes_of(self.d_o)) if planes else (self.d_o, None)
        b.bt_op_attention_mod_bwd(*x, self.o.reshape(B * T, C).float().contiguous(), self.lse.float().contiguous(), *g, B, T, C, H,
                                  self.mod, dqkv, split, self.scratch, self.scratch.numel(), flags)
        b.bt_op_attention_mod_check(self.scratch)
        assert (guard[0] == 7).all() and (guard[-1] == 7).all()
        if planes_out:
            check_split(split, dqkv.cpu().numpy())
        return dqkv

    def check(self, planes, flags=0, planes_out=False, tol=TOL):
        o, lse = self.forward(planes, flags, planes_out)
        assert close(o.view_as(self.o), self.o, tol), "o"
        empty = self.lse == -math.inf
        assert torch.equal(lse == -math.inf, empty)
        # an lse is a sum of scores: its error is that of a score (see the module's text), absolute
        assert ((lse.double() - self.lse)[~empty].abs() <= tol * (1 + self.lse[~empty].abs())).all(), "lse"
        rows = empty.permute(0, 2, 1)[..., None]
        assert (o.view_as(self.o)[rows.expand_as(self.o)] == 0).all()
        dqkv = self.backward(planes, flags, planes_out).view_as(self.grad)
        for n, name in enumerate("qkv"):
            assert close(dqkv[:, :, n], self.grad[:, :, n], tol, self.size[n]), "d" + name
        assert (dqkv[:, :, 0][rows.expand_as(self.o)] == 0).all()


def close(got, want, tol, size=0.0):
    """`size`: the norm of what was added up, where the result may have cancelled."""
    return float((got.double() - want).norm()) <= tol * max(float(want.norm()), size)


def see_fast(doc, mark, window, B, T):
    see = np.zeros((B, T, T), bool)
    i = np.arange(T)
    for n in range(B):
        ids, marks = np.zeros(T, int) if doc is None else doc[n], np.zeros(T, int) if mark is None else mark[n]
        cuts = [0] + list(np.flatnonzero(np.diff(ids)) + 1) + [T]
        for s, e in zip(cuts[:-1], cuts[1:]):
            if ids[s] < 0:
                continue
            p = s + (int(np.argmin(marks[s:e] != 0)) if (marks[s:e] == 0).any() else e - s)
            m = (i[None, s:e] <= i[s:e, None]) | (i[None, s:e] < p)
            if window:
                m &= i[s:e, None] - i[None, s:e] < window
            see[n, s:e, s:e] = m
    return see


def ways(d):
    """(planes, flags) of every kernel family that serves this head_dim."""
    out = [(False, b.BT_FLAG_ATTN_SIMT), (False, 0)]
    return out + ([(True, 0)] if d >= 64 else [])


MODS = [
    dict(),
    dict(cap=30.0),
    dict(cap=2.0, scale=1.5),                      # deep in the bend of the tanh
    dict(slope=True),
    dict(mean=40, slope=True),
    dict(mean=30, pad=50, cap=20.0),               # padding inside and at the end: empty rows
    dict(mean=70, prefix=25),
    dict(mean=70, prefix=25, window=17, slope=True, cap=50.0),
    dict(window=1),
    dict(window=100),
]


@gpu
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("mod", range(len(MODS)))
def test_attention_mod_modifications(d, mod):
    case = Case(2, 200, 3, d, seed=mod, **MODS[mod])
    for planes, flags in ways(d):
        case.check(planes, flags, planes_out=mod % 2 == 0)


@gpu
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("T", [1, 2, 31, 63, 64, 65, 127, 128, 129, 193, 257, 333])
def test_attention_mod_lengths(d, T):
    for k, mod in enumerate((dict(), dict(mean=max(1, T // 3), pad=T // 4, prefix=T // 8, slope=True, cap=30.0))):
        case = Case(1 + T % 3, T, 2, d, seed=T + k, **mod)
        for planes, flags in ways(d):
            case.check(planes, flags)


@gpu
@pytest.mark.parametrize("d", [16, 64, 128])
def test_attention_mod_rows_that_read_nothing(d):
    """All padding; one live document between padding; documents of one position."""
    T = 300
    for k, doc in enumerate((np.full((2, T), -1), np.where((np.arange(T) // 100 == 1)[None], 3, -2).repeat(2, 0),
                             np.arange(T)[None].repeat(2, 0))):
        case = Case(2, T, 2, d, seed=k, doc=doc.astype(np.int32), cap=30.0, slope=True)
        for planes, flags in ways(d):
            case.check(planes, flags, planes_out=True)


@gpu
@pytest.mark.parametrize("d", [32, 64, 128])
def test_attention_mod_large_and_small_scores(d):
    """Scores of hundreds (one key takes a row) and of 1e-6 (the cap's linear part).  A score s carries an error of
    up to 3e-6 |s| / 2 (the module's text), which is what the probabilities of the large scores may be off by."""
    for scale, cap, tol in ((6.0, 0.0, 2e-4), (6.0, 50.0, 2e-4), (1e-3, 30.0, TOL)):
        case = Case(1, 150, 2, d, cap=cap, scale=scale, seed=3)
        for planes, flags in ways(d):
            case.check(planes, flags, tol=tol)


@gpu
@pytest.mark.parametrize("B,T,H,d,mod", [
    (1, 2100, 2, 64, dict(mean=700, cap=30.0)), (1, 4097, 1, 64, dict(slope=True)), (2, 1025, 3, 128, dict(mean=500, prefix=90)),
    (1, 4097, 1, 128, dict()), (1, 4097, 1, 32, dict(cap=50.0)), (3, 777, 2, 16, dict(mean=100, pad=200, slope=True)),
    (1, 8192, 1, 64, dict())])
def test_attention_mod_long(B, T, H, d, mod):
    case = Case(B, T, H, d, seed=11, **mod)
    for planes, flags in ways(d):
        if not flags:
            case.check(planes, flags)


@gpu
@pytest.mark.parametrize("B,H", [(1, 1), (5, 7), (2, 160)])
def test_attention_mod_many_heads(B, H):
    """Grids of less than one and of several rounds over the SMs, with an odd number of heads."""
    case = Case(B, 140, H, 64, seed=B, mean=60, slope=True)
    case.check(True)
    case.check(False)


@gpu
@pytest.mark.parametrize("d", [32, 64, 128])
def test_attention_mod_same_bits_every_time(d):
    case = Case(2, 333, 3, d, mean=100, pad=50, prefix=20, cap=30.0, slope=True)
    for planes, flags in ways(d):
        first = [t.clone() for t in (*case.forward(planes, flags), case.backward(planes, flags))]
        for _ in range(3):
            for x, y in zip(first, (*case.forward(planes, flags), case.backward(planes, flags))):
                assert torch.equal(x, y)


@gpu
@pytest.mark.parametrize("d", [32, 64, 128])
def test_attention_mod_gradient_against_differences(d):
    """Directional derivative of sum(o * g): (f(x + h u) - f(x - h u)) / 2h.  With h = 2^-6 and scores of order one the
    cubic term is below h^2 = 2.5e-4 of the derivative's scale, the outputs' 1e-5 over h about the same again."""
    case = Case(1, 150, 2, d, mean=60, prefix=10, cap=5.0, slope=True)
    planes = d >= 64
    u = torch.randn(case.qkv.shape, generator=torch.Generator(DEV).manual_seed(9), device=DEV)
    h = 2.0 ** -6
    base, f = case.qkv, []
    grad = case.backward(planes).double()
    for sign in (1.0, -1.0):
        case.qkv = base + sign * h * u
        f.append(float((case.forward(planes)[0].double() * case.d_o.double()).sum()))
    want = float((grad * u.double()).sum())
    assert abs((f[0] - f[1]) / (2 * h) - want) <= 2e-3 * float(grad.norm() * u.double().norm()) / math.sqrt(grad.numel()) * 10


@gpu
@pytest.mark.parametrize("d", [32, 64, 128])
def test_attention_mod_captured_and_replayed(d):
    """A captured step gives the eager step's bits, also for inputs and spans written after the capture."""
    planes = d >= 64
    a, c = (Case(2, 260, 2, d, seed=s, mean=90, pad=30, cap=30.0, slope=True) for s in (1, 50))
    B, T, C, H = a.B, a.T, a.C, a.H
    want = [(*k.forward(planes), k.backward(planes)) for k in (a, c)]
    pack = (lambda t: planes_of(t)) if planes else (lambda t: t.clone())
    x, g, spans = pack(a.qkv), pack(a.d_o), a.spans.clone()
    o_in, lse_in = a.o.reshape(B * T, C).float().contiguous(), a.lse.float().contiguous()
    mod = b.make_attn_mod(30.0, a.slopes, spans)
    o, lse, dqkv = torch.empty(B * T, C, device=DEV), torch.empty(B, H, T, device=DEV), torch.empty(B * T, 3 * C, device=DEV)
    arg = lambda t: (None, t) if planes else (t, None)  # noqa: E731

    def step():
        b.bt_op_attention_mod_fwd(*arg(x), B, T, C, H, mod, o, None, lse, a.scratch, a.scratch.numel())
        b.bt_op_attention_mod_bwd(*arg(x), o_in, lse_in, *arg(g), B, T, C, H, mod, dqkv, None, a.scratch, a.scratch.numel())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    for k, w in ((a, want[0]), (c, want[1]), (a, want[0])):
        x.copy_(pack(k.qkv)), g.copy_(pack(k.d_o)), spans.copy_(k.spans)
        o_in.copy_(k.o.reshape(B * T, C)), lse_in.copy_(k.lse)
        o.fill_(7.0), dqkv.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, w[0]) and torch.equal(lse, w[1]) and torch.equal(dqkv, w[2])


@gpu
def test_attention_mod_two_streams():
    cases = [Case(2, 500, 4, 64, seed=s, mean=200, cap=30.0) for s in (1, 2)]
    want = [(*k.forward(True), k.backward(True)) for k in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        got = []
        for k, s in zip(cases, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                B, T, C, H = k.B, k.T, k.C, k.H
                o, lse, dqkv = torch.empty(B * T, C, device=DEV), torch.empty(B, H, T, device=DEV), torch.empty(B * T, 3 * C, device=DEV)
                x, g = planes_of(k.qkv), planes_of(k.d_o)
                o_in, lse_in = k.o.reshape(B * T, C).float().contiguous(), k.lse.float().contiguous()
                b.bt_op_attention_mod_fwd(None, x, B, T, C, H, k.mod, o, None, lse, k.scratch, k.scratch.numel())
                b.bt_op_attention_mod_bwd(None, x, o_in, lse_in, None, g, B, T, C, H, k.mod, dqkv, None, k.scratch, k.scratch.numel())
                got.append((o, lse, dqkv, x, g, o_in, lse_in))
        torch.cuda.synchronize()
        for w, g in zip(want, got):
            assert all(torch.equal(p, q) for p, q in zip(w, g))


@gpu
@pytest.mark.parametrize("d", [16, 32, 64, 128])
def test_attention_mod_softcaps_at_the_ends_of_the_range(d):
    """1e-20: every score is worth nothing, rows are plain means and pass no gradient on to q and k.  1e20: no cap at all."""
    for cap in (1e-20, 1e20):
        for T in (60, 270):
            case = Case(1, T, 2, d, cap=cap, seed=T)
            for planes, flags in ways(d):
                case.check(planes, flags)


@gpu
@pytest.mark.parametrize("d,T", [(16, 100), (16, 300), (32, 100), (32, 200), (64, 200), (128, 140)])
def test_attention_mod_every_form_of_the_inputs(d, T):
    """qkv and d_o raw, as planes, and both, in every combination; the scratch holds anything."""
    case = Case(2, T, 2, d, seed=d, mean=80, pad=20, cap=30.0, slope=True)
    B, C, H = case.B, case.C, case.H
    o, lse = case.o.reshape(B * T, C).float().contiguous(), case.lse.float().contiguous()
    for x in ((case.qkv, None), (None, planes_of(case.qkv)), (case.qkv, planes_of(case.qkv))):
        out, got = torch.empty(B * T, C, device=DEV), torch.empty(B, H, T, device=DEV)
        b.bt_op_attention_mod_fwd(*x, B, T, C, H, case.mod, out, None, got, case.scratch, case.scratch.numel())
        assert close(out.view_as(case.o), case.o, TOL)
        for g in ((case.d_o, None), (None, planes_of(case.d_o)), (case.d_o, planes_of(case.d_o))):
            case.scratch.fill_(255)
            dqkv = torch.empty(B * T, 3 * C, device=DEV)
            b.bt_op_attention_mod_bwd(*x, o, lse, *g, B, T, C, H, case.mod, dqkv, None, case.scratch, case.scratch.numel())
            b.bt_op_attention_mod_check(case.scratch)
            for n in range(3):
                assert close(dqkv.view_as(case.grad)[:, :, n], case.grad[:, :, n], TOL, case.size[n])


def off16(*shape):
    """An array that starts 16 bytes behind a 32-byte boundary."""
    n = math.prod(shape)
    t = torch.empty(n + 8, device=DEV)[4:4 + n].view(shape)
    assert t.data_ptr() % 32 == 16
    return t


@gpu
@pytest.mark.parametrize("d,T", [(16, 300), (32, 60), (32, 200), (64, 200), (128, 140)])
def test_attention_mod_arrays_on_16_bytes(d, T):
    """Arrays need 16-byte alignment only: the same bits as from 32-byte aligned ones."""
    case = Case(2, T, 3, d, seed=5, cap=30.0, mean=70)
    B, C, H = case.B, case.C, case.H
    o, lse = case.o.reshape(B * T, C).float().contiguous(), case.lse.float().contiguous()
    for planes in ((False, True) if d >= 64 else (False,)):
        got = []
        for new in (lambda *s: torch.empty(*s, device=DEV), off16):
            put = lambda t: new(*t.shape).copy_(t)  # noqa: B023,E731
            x = (None, put(planes_of(case.qkv))) if planes else (put(case.qkv), None)
            g = (None, put(planes_of(case.d_o))) if planes else (put(case.d_o), None)
            out, out2, l2 = new(B * T, C), new(2, B * T, C), new(B, H, T)
            dx, dx2 = new(B * T, 3 * C), new(2, B * T, 3 * C)
            b.bt_op_attention_mod_fwd(*x, B, T, C, H, case.mod, out, out2, l2, case.scratch, case.scratch.numel())
            b.bt_op_attention_mod_bwd(*x, put(o), put(lse), *g, B, T, C, H, case.mod, dx, dx2, case.scratch, case.scratch.numel())
            got.append((out, out2, l2, dx, dx2))
        assert all(torch.equal(p, q) for p, q in zip(*got))
        assert close(got[1][0].view_as(case.o), case.o, TOL)


@gpu
@pytest.mark.parametrize("d,planes", [(16, False), (32, True), (64, False), (64, True), (128, True)])
def test_attention_mod_more_heads_than_a_grid_axis(d, planes):
    """65,600 sequences of three positions; they are alike, so the answer is that of one."""
    B, T = 65600, 3
    one = Case(1, T, 1, d, cap=20.0, seed=3)
    arg = (lambda t: (None, planes_of(t))) if planes else (lambda t: (t, None))
    o, lse = torch.empty(B * T, d, device=DEV), torch.empty(B, 1, T, device=DEV)
    size = b.bt_op_attention_mod_scratch_bytes(B, T, d, 1)
    scratch, mod, dqkv = torch.empty(size, dtype=torch.uint8, device=DEV), b.make_attn_mod(20.0), torch.empty(B * T, 3 * d, device=DEV)
    x, g = arg(one.qkv.repeat(B, 1)), arg(one.d_o.repeat(B, 1))
    b.bt_op_attention_mod_fwd(*x, B, T, d, 1, mod, o, None, lse, scratch, size)
    b.bt_op_attention_mod_bwd(*x, o, lse, *g, B, T, d, 1, mod, dqkv, None, scratch, size)
    b.bt_op_attention_mod_check(scratch)
    for all_, first, want in ((o, o[:T], one.o), (dqkv, dqkv[:T], one.grad)):
        assert torch.equal(all_.view(B, T, -1), first[None].expand(B, -1, -1))
        assert close(first.view_as(want), want, TOL, sum(one.size))


@gpu
def test_attention_mod_narrow_heads_on_two_streams():
    """Heads of 32 go through planes in the call's own scratch: two calls at once do not meet."""
    cases = [Case(2, 400, 4, 32, seed=s, mean=200, cap=30.0) for s in (1, 2)]
    want = [(*k.forward(False), k.backward(False)) for k in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        got = []
        for k, s in zip(cases, streams):
            s.wait_stream(torch.cuda.current_stream())
            B, T, C, H = k.B, k.T, k.C, k.H
            o, lse, dqkv = torch.empty(B * T, C, device=DEV), torch.empty(B, H, T, device=DEV), torch.empty(B * T, 3 * C, device=DEV)
            o_in, lse_in = k.o.reshape(B * T, C).float().contiguous(), k.lse.float().contiguous()
            torch.cuda.synchronize()
            # the stream by name, not as the current one
            b.bt_op_attention_mod_fwd(k.qkv, None, B, T, C, H, k.mod, o, None, lse, k.scratch, k.scratch.numel(), stream=s.cuda_stream)
            b.bt_op_attention_mod_bwd(k.qkv, None, o_in, lse_in, k.d_o, None, B, T, C, H, k.mod, dqkv, None, k.scratch,
                                      k.scratch.numel(), stream=s.cuda_stream)
            got.append((o, lse, dqkv, o_in, lse_in))
        torch.cuda.synchronize()
        for w, g in zip(want, got):
            assert all(torch.equal(p, q) for p, q in zip(w, g))


@gpu
@pytest.mark.parametrize("d,planes", [(32, False), (64, True), (128, True)])
def test_attention_mod_past_two_to_the_31_elements(d, planes):
    """1,000 sequences of 1,000 positions: qkv alone has 2.3e9 elements.  All are alike, so the answer is that of one."""
    B, T, C = 1000, 1000, 768
    H = C // d
    one = Case(1, T, H, d, cap=20.0, seed=3, mean=300)
    spans = spans_of(random_layout(np.random.default_rng(3 + 7 * T), 1, T, 300, 0, 0)[0].repeat(B, 0), None, 0, B, T)
    mod, size = b.make_attn_mod(20.0, None, spans), b.bt_op_attention_mod_scratch_bytes(B, T, C, H)
    scratch = torch.empty(size, dtype=torch.uint8, device=DEV)
    if planes:
        arg = lambda t: (None, planes_of(t)[:, None].expand(2, B, *t.shape).contiguous())  # noqa: E731
    else:
        arg = lambda t: (t.repeat(B, 1), None)  # noqa: E731
    x = arg(one.qkv)
    o, lse = torch.empty(B, T, C, device=DEV), torch.empty(B, H, T, device=DEV)
    b.bt_op_attention_mod_fwd(*x, B, T, C, H, mod, o, None, lse, scratch, size)
    assert close(o[0].view_as(one.o), one.o, TOL)
    assert all(torch.equal(o[n], o[0]) for n in range(B)) and torch.equal(lse, lse[:1].expand_as(lse))
    g, dqkv = arg(one.d_o), torch.empty(B, T, 3 * C, device=DEV)
    b.bt_op_attention_mod_bwd(*x, o, lse, *g, B, T, C, H, mod, dqkv, None, scratch, size)
    b.bt_op_attention_mod_check(scratch)
    assert close(dqkv[0].view_as(one.grad), one.grad, TOL, sum(one.size))
    assert all(torch.equal(dqkv[n], dqkv[0]) for n in range(B))


@gpu
def test_rope_and_dropout_past_two_to_the_32_elements():
    H, d, N = 12, 64, 1_900_000
    C, cfg = H * d, b.make_rope(d)
    few = rand(1, 1000, 3 * C)
    x, want = few.repeat(N // 1000, 1), torch.empty_like(few)          # 4.4e9 elements
    b.bt_op_rope_fwd(few, None, 1000, 1000, C, H, cfg, want)
    b.bt_op_rope_fwd(x, None, N, 1000, C, H, cfg, x)
    assert all(torch.equal(part, want) for part in x.split(1000))
    n = 2 ** 32 + 1028
    x = x.view(-1)[:n].fill_(1.0)
    b.bt_op_dropout_fwd(x, None, n, 0.5, 7, 9, x)
    for at in (0, 2 ** 31 - 32, 2 ** 32 - 32, n - 64):
        assert np.array_equal(np64(x[at:at + 64]) != 0, keep_mask(64, 0.5, 7, 9, at // 4))


@gpu
@pytest.mark.parametrize("d,T", [(16, 60), (16, 300), (32, 200), (64, 200), (128, 140)])
def test_attention_mod_planes_alone_as_the_output(d, T):
    """Without a raw output the planes are those of the call that writes both."""
    case = Case(2, T, 2, d, seed=8, mean=70, pad=15, cap=30.0)
    B, C, H = case.B, case.C, case.H
    o_in, lse_in = case.o.reshape(B * T, C).float().contiguous(), case.lse.float().contiguous()
    for planes, flags in ways(d):
        x = (None, planes_of(case.qkv)) if planes else (case.qkv, None)
        g = (None, planes_of(case.d_o)) if planes else (case.d_o, None)
        got = []
        for raw in (True, False):
            o, dx = (torch.empty(B * T, C, device=DEV), torch.empty(B * T, 3 * C, device=DEV)) if raw else (None, None)
            o2, dx2, lse = torch.empty(2, B * T, C, device=DEV), torch.empty(2, B * T, 3 * C, device=DEV), torch.empty(B, H, T, device=DEV)
            b.bt_op_attention_mod_fwd(*x, B, T, C, H, case.mod, o, o2, lse, case.scratch, case.scratch.numel(), flags)
            b.bt_op_attention_mod_bwd(*x, o_in, lse_in, *g, B, T, C, H, case.mod, dx, dx2, case.scratch, case.scratch.numel(), flags)
            got.append((o2, dx2, lse))
        assert all(torch.equal(p, q) for p, q in zip(*got))
        assert close(got[1][0].sum(0).view_as(case.o), case.o, TOL)


@gpu
def test_attention_mod_from_several_host_threads():
    cases = [Case(2, 300, 3, d, seed=d, mean=100, cap=30.0) for d in (32, 64, 128, 64)]
    want = [(*k.forward(k.d >= 64), k.backward(k.d >= 64)) for k in cases]
    bad = []

    def work(k, w):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(10):
                    if not all(torch.equal(p, q) for p, q in zip(w, (*k.forward(k.d >= 64), k.backward(k.d >= 64)))):
                        bad.append(k.d)
        except Exception as e:  # noqa: BLE001
            bad.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=a) for a in zip(cases, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad, bad


@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_attention_mod_scratch_of_calls_given_planes(d):
    """They need the error word and the row sums only; the bytes behind those stay as they were."""
    case = Case(3, 150, 2, d, seed=4, cap=30.0, mean=60)
    B, T, C, H = case.B, case.T, case.C, case.H
    small = 256 + (4 * B * H * T + 255) // 256 * 256
    buf = torch.full((small + 4096,), 77, dtype=torch.uint8, device=DEV)
    x, g = planes_of(case.qkv), planes_of(case.d_o)
    o, lse, dqkv = torch.empty(B * T, C, device=DEV), torch.empty(B, H, T, device=DEV), torch.empty(B * T, 3 * C, device=DEV)
    b.bt_op_attention_mod_fwd(None, x, B, T, C, H, case.mod, o, None, lse, buf, small)
    b.bt_op_attention_mod_bwd(None, x, o, lse, None, g, B, T, C, H, case.mod, dqkv, None, buf, small)
    b.bt_op_attention_mod_check(buf)
    assert (buf[small:] == 77).all()
    for n in range(3):
        assert close(dqkv.view_as(case.grad)[:, :, n], case.grad[:, :, n], TOL, case.size[n])
    with pytest.raises(b.BtError):
        b.bt_op_attention_mod_bwd(None, x, o, lse, case.d_o, None, B, T, C, H, case.mod, dqkv, None, buf, small)
    with pytest.raises(b.BtError):
        b.bt_op_attention_mod_fwd(None, x, B, T, C, H, case.mod, o, None, lse, buf, small - 1)


@gpu
def test_attention_mod_plain_equals_causal_attention():
    """Without a modification the operator is the causal attention beside it."""
    B, T, H, d = 2, 300, 3, 64
    case = Case(B, T, H, d)
    o, lse = case.forward(True)
    ref, ref_lse = torch.empty(B * T, H * d, device=DEV), torch.empty(B, H, T, device=DEV)
    b.bt_op_attention_fwd(None, B, T, H * d, H, ref, None, ref_lse, qkv_split=planes_of(case.qkv))
    assert rel_l2(np64(o), np64(ref)) < TOL and rel_l2(np64(lse), np64(ref_lse)) < TOL


# ------------------------------------------------------------------------------- dropout

@gpu
@pytest.mark.parametrize("n,p,seed,offset", [
    (1, 0.5, 0, 0), (3, 0.5, 1, 1), (4, 0.1, 7, 5), (5, 0.1, 2 ** 63 + 5, 2 ** 40 + 3), (768, 0.0, 3, 1), (1023, 0.9, 3, 2 ** 64 - 1),
    (16384, 0.25, 123456789, 3), (20002, 0.1, 5, 9)])
def test_dropout(n, p, seed, offset):
    keep = keep_mask(n, p, seed, offset)
    scale = float(np.float32(1.0 / (1.0 - p)))
    x, res = rand(1, n), rand(2, n)
    buf = torch.full((n + 16,), 7.0, device=DEV)
    y = buf[4:4 + n]
    b.bt_op_dropout_fwd(x, res, n, p, seed, offset, y)
    want = np.where(keep, np64(x) * scale, 0.0) + np64(res)
    # one rounding of the product and one of the sum
    assert (np.abs(np64(y) - want) <= 2.0 ** -24 * (np.abs(np64(x)) * scale + np.abs(want)) + 1e-30).all()
    assert (buf[:4] == 7).all() and (buf[4 + n:] == 7).all()
    b.bt_op_dropout_fwd(x, None, n, p, seed, offset, y)
    assert np.array_equal(np64(y), np.where(keep, (x * scale).cpu().numpy(), 0.0))
    dx = torch.empty(n, device=DEV)
    b.bt_op_dropout_bwd(x, n, p, seed, offset, dx)
    assert torch.equal(dx, y)                                    # same mask, same factor
    same = x.clone()
    b.bt_op_dropout_fwd(same, None, n, p, seed, offset, same)    # in place
    assert torch.equal(same, y)
    if n % 4 == 0:
        planes = torch.empty(2, n, device=DEV)
        b.bt_op_dropout_bwd(x, n, p, seed, offset, None, planes)
        check_split(planes, dx.cpu().numpy())


@gpu
def test_dropout_hides_what_it_drops_and_keeps_the_share():
    n, p = 1 << 20, 0.3
    x = torch.full((n,), math.nan, device=DEV)
    y = torch.empty(n, device=DEV)
    b.bt_op_dropout_fwd(x, None, n, p, 11, 0, y)
    kept = ~(y == 0)
    assert torch.equal(torch.isnan(y), kept)
    share = float(kept.double().mean())
    assert abs(share - (1 - p)) < 6 * math.sqrt(p * (1 - p) / n)     # six standard deviations
    z = torch.empty(n, device=DEV)
    b.bt_op_dropout_fwd(x, None, n, p, 11, 1, z)                     # another offset, another mask
    both = float((kept & ~(z == 0)).double().mean())
    assert abs(both - (1 - p) ** 2) < 6 * math.sqrt((1 - p) ** 2 / n)


@gpu
def test_dropout_captured_with_a_step_word():
    n, p = 4096, 0.2
    x, y = rand(1, n), torch.empty(n, device=DEV)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    step16 = torch.zeros(2, dtype=torch.int64, device=DEV)[:1]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.bt_op_dropout_fwd(x, None, n, p, 5, 100, y, d_step=step16)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            b.bt_op_dropout_fwd(x, None, n, p, 5, 100, y, d_step=step)
            step.add_(1)
    want = torch.empty(n, device=DEV)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        b.bt_op_dropout_fwd(x, None, n, p, 5, 100 + k, want)
        assert torch.equal(y, want)


# ------------------------------------------------------------------------------- together

@gpu
@pytest.mark.parametrize("d", [32, 64, 128])
def test_sublayer_forward_and_backward(d):
    """qkv -> rotation -> attention over packed documents -> dropout and residual, and back."""
    B, T, H, p, seed = 2, 190, 3, 0.15, 77
    C, n, planes = H * d, B * T, d >= 64
    doc, mark = random_layout(np.random.default_rng(4), B, T, 60, 20, 9)
    pos = np.zeros((B, T), np.int32)
    for s in range(B):
        for i in range(1, T):
            pos[s, i] = pos[s, i - 1] + 1 if doc[s, i] == doc[s, i - 1] else 0
    qkv, resid, dy = rand(1, n, 3 * C), rand(2, n, C), rand(3, n, C)
    slopes = torch.tensor([0.5 / (h + 1) for h in range(H)], device=DEV)
    spans = spans_of(doc, mark, 0, B, T)
    mod, cfg = b.make_attn_mod(30.0, slopes, spans), b.make_rope(d // 2, mscale=1.1)
    pos_d = torch.tensor(pos.reshape(-1), device=DEV)
    scratch = torch.empty(b.bt_op_attention_mod_scratch_bytes(B, T, C, H), dtype=torch.uint8, device=DEV)
    new = lambda *s: torch.empty(*s, device=DEV)  # noqa: E731
    rot, o, lse, y = new(2, n, 3 * C) if planes else new(n, 3 * C), new(n, C), new(B, H, T), new(n, C)
    b.bt_op_rope_fwd(qkv, pos_d, n, T, C, H, cfg, None if planes else rot, rot if planes else None)
    arg = (lambda t: (None, t)) if planes else (lambda t: (t, None))
    b.bt_op_attention_mod_fwd(*arg(rot), B, T, C, H, mod, o, None, lse, scratch, scratch.numel())
    b.bt_op_dropout_fwd(o, resid, n * C, p, seed, 1, y)
    d_o = new(2, n, C) if planes else new(n, C)
    b.bt_op_dropout_bwd(dy, n * C, p, seed, 1, None if planes else d_o, d_o if planes else None)
    drot, dqkv = new(n, 3 * C), new(n, 3 * C)
    b.bt_op_attention_mod_bwd(*arg(rot), o, lse, *arg(d_o), B, T, C, H, mod, drot, None, scratch, scratch.numel())
    b.bt_op_rope_bwd(drot, pos_d, n, T, C, H, cfg, dqkv)
    b.bt_op_attention_mod_check(scratch)

    theta, m = thetas(d // 2), float(np.float32(1.1))
    x = torch.tensor(rope64(np64(qkv), pos.reshape(-1), H, d // 2, False, theta, m), device=DEV)
    keep = torch.tensor(keep_mask(n * C, p, seed, 1), device=DEV).view(n, C) / (1 - p)
    see = torch.tensor(see_matrix(doc, mark, 0, B, T), device=DEV)
    ref_o, _, grad, _ = attention64(x.view(B, T, 3, H, d), see, 30.0, slopes.double(), (dy.double() * keep).view(B, T, H, d))
    assert rel_l2(np64(y), np64(ref_o.reshape(n, C) * keep + resid.double())) < TOL
    want = rope64(np64(grad.reshape(n, 3 * C)), pos.reshape(-1), H, d // 2, False, theta, m, -1.0)
    assert rel_l2(np64(dqkv), want) < TOL
