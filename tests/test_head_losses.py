"""Cross entropy and distillation at the language-model head without the logits, and distillation on logits,
against plain 64-bit forms.

Tolerances.  Half a rounding of an FP32 value is 2^-24 of it.  A score of the tensor-core kernels is a sum of products of
FP16 pairs: each operand is held to 2^-23 of itself, the dropped product of the low halves is 2^-24 of a product, and the
accumulator truncates, by at most 2^-23 of the running sum per instruction, 96 instructions between two sums in registers:
96 * 2^-23 = 1.1e-5 of a partial score, half of that on average and less where partial sums change sign.  A score error e
moves a probability by e, so with scores of a few units losses are within 2e-5 and gradients within 2e-5 of their norm;
the plain FP32 kernels are well inside that.
"""
import math

import numpy as np
import pytest
import torch

from paper_2606_24780_b200 import binding as b
from paper_2606_24780_b200 import build as bt_build

from gpu_util import DEV, check_split

gpu = pytest.mark.gpu
TOL = 2e-5


# ------------------------------------------------------------------------------- 64-bit forms

def aims64(N, V, targets=None, ids=None, top=None, tau=1.0, lse=None):
    """Dense aims [N, V] and sum_k p log p [N] from the definition, entry by entry; numpy, 64 bits."""
    a, h = np.zeros((N, V)), np.zeros(N)
    for n in range(N):
        if targets is not None:
            if targets[n] >= 0:
                a[n, targets[n] if targets[n] < V else 0] = 1.0
            continue
        there = [(int(i) if i < V else 0, float(t) / tau) for i, t in zip(ids[n], top[n]) if i >= 0 and t != -math.inf]
        if not there:
            continue
        most = max(t for _, t in there)
        norm = float(lse[n]) if lse is not None else most + math.log(sum(math.exp(t - most) for _, t in there))
        for i, t in there:
            a[n, i] += math.exp(t - norm)
            h[n] += math.exp(t - norm) * (t - norm)
    return a, h


def head64(z, a, h, tau, w, inv, lse=None):
    """Losses, lse, mean and the gradient at tau z of scores z = logits / tau (torch, 64 bits)."""
    own = torch.logsumexp(z, 1)
    S = a.sum(1)
    losses = torch.where(S > 0, tau ** 2 * (h + S * own - torch.where(a != 0, a * z, 0.0).sum(1)), 0.0)
    g = inv * tau * w
    live = (S > 0) & (w != 0)
    q = torch.softmax(z, 1) if lse is None else torch.exp(z - lse[:, None])
    d = g[:, None] * (q * S[:, None] - a)
    d = torch.where(live[:, None], d, 0.0)
    return losses, own, inv * torch.where(live, w * losses, 0.0).sum(), d


def rel(got, want):
    got, want = got.double().cpu(), want.double().cpu()
    n = float(want.norm())
    return float((got - want).norm()) / (n if n else 1.0)


def split(x):
    hi = ((x.view(torch.int32) + 0x1000) & ~0x1FFF).view(torch.float32)
    return torch.stack((hi, x - hi)).contiguous()


class Case:
    """Inputs of one call, and the 64-bit results for them."""

    def __init__(self, N, C, V, K=0, tau=1.0, whole=False, weights=False, pad=0, planes=False, seed=0, scale=2.0):
        rng = np.random.default_rng(seed)
        self.N, self.C, self.V, self.K, self.tau = N, C, V, K, tau
        self.inv = 1.0 / max(1, N)
        self.x = torch.tensor(rng.standard_normal((N, C)), dtype=torch.float32, device=DEV)
        self.w = torch.tensor(rng.standard_normal((V, C)) * scale / math.sqrt(C), dtype=torch.float32, device=DEV)
        self.planes = planes
        self.rw = torch.tensor(rng.uniform(0.2, 2.0, N), dtype=torch.float32, device=DEV) if weights else None
        if weights and N > 2:
            self.rw[2] = 0.0
        self.targets = self.ids = self.top = self.top_lse = None
        if K:
            ids = rng.integers(0, V, (N, K))                       # with repetition
            top = 3.0 * rng.standard_normal((N, K))
            if K > 1:
                ids[::3, 1] = ids[::3, 0]
                top[1::4, K - 1] = -math.inf
                ids[2::5, 0] = -1
            if pad:
                ids[:pad] = -1
            self.ids = torch.tensor(ids, dtype=torch.int32, device=DEV)
            self.top = torch.tensor(top, dtype=torch.float32, device=DEV)
            if whole:
                self.top_lse = torch.logsumexp(self.top.double() / tau, 1).float().nan_to_num(neginf=0.0) + 0.25
        else:
            t = rng.integers(0, V, N)
            t[:pad] = -1
            self.targets = torch.tensor(t, dtype=torch.int32, device=DEV)

    def aims(self):
        c = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
        a, h = aims64(self.N, self.V, c(self.targets), c(self.ids), c(self.top), self.tau, c(self.top_lse))
        return torch.tensor(a, device=DEV), torch.tensor(h, device=DEV)

    def weight(self):
        return torch.ones(self.N, dtype=torch.float64, device=DEV) if self.rw is None else self.rw.double()

    def want(self, lse=None):
        z = self.x.double() @ self.w.double().T / self.tau
        losses, own, mean, d = head64(z, *self.aims(), self.tau, self.weight(), self.inv, None if lse is None else lse.double())
        return losses, own, mean, d @ self.w.double(), d.T @ torch.where(d.abs().sum(1, keepdim=True) > 0, self.x.double(), 0.0)

    def sizes(self, lse):
        """Norms of dx and dw with their two terms added instead of subtracted, as those of each term."""
        a, _ = self.aims()
        q = torch.exp(self.x.double() @ self.w.double().T / self.tau - lse.double()[:, None]) * a.sum(1, keepdim=True)
        g = (self.inv * self.tau * self.weight())[:, None]
        terms = [torch.where(a.sum(1, keepdim=True) > 0, g * t, 0.0) for t in (q, a)]
        x = torch.where(a.sum(1, keepdim=True) > 0, self.x.double(), 0.0)
        return [sum(float((t @ self.w.double()).norm()) for t in terms) + 1e-300, sum(float((t.T @ x).norm()) for t in terms) + 1e-300]

    def aim(self):
        return b.make_distill(self.ids, self.top, self.tau, self.top_lse) if self.K else self.targets

    def operands(self):
        return (None, split(self.x), None, split(self.w)) if self.planes else (self.x, None, self.w, None)

    def forward(self, bad=None, scratch=None):
        N, C, V = self.N, self.C, self.V
        out = [torch.full((max(1, n),), math.nan, device=DEV) for n in (N, N, 1)]
        work = scratch if scratch is not None else torch.full((b.bt_op_head_fwd_scratch_bytes(N, C, V, self.K),), 255, dtype=torch.uint8, device=DEV)
        call = b.bt_op_head_distill_fwd if self.K else b.bt_op_head_xent_fwd
        call(*self.operands(), self.aim(), self.rw, N, C, V, self.inv, *out, work, work.numel(), bad)
        if N:
            b.bt_op_head_check(work)
        return out

    def backward(self, lse, piece=0, dx=True, dw=True, dx_split=False):
        N, C, V = self.N, self.C, self.V
        new = lambda *s: torch.full(s, math.nan, device=DEV)  # noqa: E731
        gx, gw, gs = new(N, C) if dx else None, new(V, C) if dw else None, new(2, N, C) if dx_split else None
        work = torch.full((b.bt_op_head_bwd_scratch_bytes(N, C, V, self.K, piece),), 255, dtype=torch.uint8, device=DEV)
        call = b.bt_op_head_distill_bwd if self.K else b.bt_op_head_xent_bwd
        call(*self.operands(), self.aim(), self.rw, lse, N, C, V, self.inv, gx, gw, work, work.numel(), piece, gs)
        if N:
            b.bt_op_head_check(work)
        return gx, gw, gs


def check(c, piece=0):
    losses, lse, mean = c.forward()
    want = c.want()
    top = max(1.0, float(want[1].abs().max()))
    assert float((losses - want[0]).abs().max()) < TOL * c.tau ** 2 * top
    assert float((lse - want[1]).abs().max()) < TOL * top
    assert abs(float(mean[0]) - float(want[2])) < TOL * c.tau ** 2 * top * float(c.weight().mean())
    want = c.want(lse)
    dx, dw, _ = c.backward(lse, piece)
    # S q - a is a difference: a score error e, and lse's own rounding, make an error e S q of it, relative to the two terms
    # and not to what is left of them (with one class the exact difference is lse's rounding alone, 2^-24 of q = a = 1)
    size = c.sizes(lse)
    assert float((dx - want[3]).norm()) < TOL * size[0] and float((dw - want[4]).norm()) < TOL * size[1]
    assert not dx[want[3].abs().sum(1) == 0].any()                # rows without part in the loss: exactly zero
    return losses, lse, mean, dx, dw


# ------------------------------------------------------------------------------- CPU: refusals

@pytest.fixture(scope="module")
def lib():
    bt_build.build()
    return b.lib()


def refused(fn, *args, status=1, word=""):
    with pytest.raises(b.BtError) as e:
        fn(*args)
    assert e.value.status == status and word in str(e.value), str(e.value)


def test_refusals_of_the_head_calls(lib):
    P = 0x10000                                                   # never read: every call is refused on the host

    def fwd(x=P, xs=None, w=P, ws=None, t=P, rw=None, N=4, C=64, V=100, losses=2 * P, lse=None, mean=None, scratch=3 * P, size=1 << 40, bad=None):
        b.bt_op_head_xent_fwd(x, xs, w, ws, t, rw, N, C, V, 1.0, losses, lse, mean, scratch, size, bad, 0)

    def bwd(x=P, w=P, t=P, lse=4 * P, N=4, C=64, V=100, dx=2 * P, dw=None, scratch=3 * P, size=1 << 40, piece=0):
        b.bt_op_head_xent_bwd(x, None, w, None, t, None, lse, N, C, V, 1.0, dx, dw, scratch, size, piece, None, 0)

    for bad in (dict(C=48), dict(C=0), dict(C=4128), dict(V=0), dict(V=(1 << 24) + 1), dict(N=-1), dict(N=(1 << 24) + 1), dict(x=None), dict(w=None),
                dict(t=None), dict(losses=None), dict(scratch=None), dict(scratch=3 * P + 128), dict(x=P + 4), dict(t=P + 4), dict(rw=P + 8),
                dict(bad=P + 2), dict(losses=P), dict(mean=P)):
        refused(lambda: fwd(**bad))
    refused(lambda: fwd(size=b.bt_op_head_fwd_scratch_bytes(4, 64, 100) - 1), status=3, word="scratch")
    for bad in (dict(lse=None), dict(dx=None), dict(piece=-1), dict(dx=P), dict(dw=4 * P), dict(dw=P + 4)):
        refused(lambda: bwd(**bad))
    refused(lambda: bwd(size=b.bt_op_head_bwd_scratch_bytes(4, 64, 100) - 1), status=3, word="scratch")
    refused(lambda: b.bt_op_head_check(None, 0))
    refused(lambda: b.bt_op_head_check(3 * P + 16, 0))
    for args in ((4, 48, 100, 0), (-1, 64, 100, 0), (4, 64, 0, 0), (4, 64, 100, 1025), (4, 64, 100, -1)):
        assert b.bt_op_head_fwd_scratch_bytes(*args) == 0 and b.bt_op_head_bwd_scratch_bytes(*args) == 0
    assert b.bt_op_head_bwd_scratch_bytes(4, 64, 100, 0, -1) == 0


def test_refusals_of_the_distillation_calls(lib):
    P = 0x10000

    def teacher(K=4, tau=1.0, ids=P, logits=P, lse=None):
        return b.bt_distill(K, tau, ids, logits, lse)

    def both(t, **kw):
        def head():
            b.bt_op_head_distill_fwd(P, None, P, None, t, None, 4, 64, 100, 1.0, 2 * P, None, None, 3 * P, 1 << 40, None, 0)

        def back():
            b.bt_op_head_distill_bwd(P, None, P, None, t, None, P, 4, 64, 100, 1.0, 2 * P, None, 3 * P, 1 << 40, 0, None, 0)

        def logits():
            b.bt_op_softmax_distill(5 * P, t, None, 4, 100, 100, 1.0, 2 * P, None, None, None, None, 0)
        for fn in (head, back, logits):
            refused(fn, **kw)

    both(None)
    for bad in (dict(K=0), dict(K=1025), dict(tau=0.0), dict(tau=-1.0), dict(tau=math.nan), dict(tau=1e5), dict(ids=None), dict(logits=None),
                dict(ids=P + 4), dict(logits=P + 8), dict(lse=P + 4)):
        both(teacher(**bad))

    def logits(z=5 * P, N=4, V=100, ld=100, losses=2 * P, mean=None, dz=None, planes=None, bad=None):
        b.bt_op_softmax_distill(z, teacher(), None, N, V, ld, 1.0, losses, mean, dz, planes, bad, 0)

    for bad in (dict(z=None), dict(z=5 * P + 4), dict(N=-1), dict(N=(1 << 24) + 1), dict(V=0), dict(ld=99), dict(V=101), dict(V=98, ld=98), dict(losses=None),
                dict(losses=P), dict(dz=P), dict(planes=5 * P - 1600), dict(bad=P + 1), dict(mean=P + 4)):
        refused(lambda: logits(**bad))


def test_teacher_arrays_of_the_wrong_shape_are_refused(lib):
    ids, top = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, 5)
    with pytest.raises(ValueError):
        b.make_distill(ids, top)
    with pytest.raises(ValueError):
        b.make_distill(ids[0], top[0])


# ------------------------------------------------------------------------------- GPU: the head

@gpu
@pytest.mark.parametrize("N,C,V", [(1, 32, 1), (1, 768, 50257), (2, 64, 31), (3, 96, 257), (5, 1024, 4099), (7, 4096, 300), (8, 64, 512),
                                   (9, 64, 513), (33, 160, 1000), (100, 768, 2049), (127, 64, 255), (128, 64, 256), (129, 96, 257),
                                   (255, 1056, 511), (256, 512, 1024), (257, 64, 1025), (300, 2080, 700), (513, 128, 3), (1000, 64, 5003),
                                   (2049, 32, 130), (16, 96, 300), (17, 32, 129), (40, 4096, 300),
                                   (200, 4096, 500), (65, 2080, 1000), (1200, 96, 40)])
@pytest.mark.parametrize("planes", [False, True])
def test_cross_entropy(N, C, V, planes):
    check(Case(N, C, V, planes=planes, weights=N % 2 == 1, pad=N // 5, seed=N + V))


@gpu
@pytest.mark.parametrize("N,C,V", [(24, 768, 50257), (100, 1024, 50257), (128, 96, 60001), (33, 2080, 40000), (11, 64, 90000)])
@pytest.mark.parametrize("planes", [False, True])
def test_some_dozens_of_rows_over_many_tiles(N, C, V, planes):
    """Several tiles of 128 rows of W to every SM, of one to 33 blocks each, several times over: every value of every run."""
    gen = torch.Generator(DEV).manual_seed(N)
    x, w = torch.randn(N, C, generator=gen, device=DEV), torch.randn(V, C, generator=gen, device=DEV) * 2 / math.sqrt(C)
    t = torch.randint(0, V, (N,), generator=gen, device=DEV, dtype=torch.int32)
    z = x.double() @ w.double().T
    want = torch.logsumexp(z, 1)
    loss = want - z.gather(1, t.long()[:, None])[:, 0]
    work = torch.empty(b.bt_op_head_fwd_scratch_bytes(N, C, V), dtype=torch.uint8, device=DEV)
    operands = (None, split(x), None, split(w)) if planes else (x, None, w, None)
    for _ in range(8):
        losses, lse = torch.full((N,), math.nan, device=DEV), torch.full((N,), math.nan, device=DEV)
        b.bt_op_head_xent_fwd(*operands, t, None, N, C, V, 1.0, losses, lse, None, work, work.numel())
        b.bt_op_head_check(work)
        assert float((lse - want).abs().max()) < TOL * 10 and float((losses - loss).abs().max()) < TOL * 10


@gpu
@pytest.mark.parametrize("N,C,V,K,tau,whole", [(1, 64, 40, 1, 1.0, False), (4, 32, 5, 16, 2.0, False), (8, 768, 3001, 64, 2.0, True),
                                               (40, 96, 999, 3, 0.5, True), (128, 128, 5000, 200, 2.0, False), (130, 64, 700, 128, 4.0, False), (260, 512, 2050, 33, 1.5, True),
                                               (300, 64, 1500, 1024, 1.0, False), (1001, 32, 257, 7, 1.0, False)])
@pytest.mark.parametrize("planes", [False, True])
def test_distillation(N, C, V, K, tau, whole, planes):
    check(Case(N, C, V, K=K, tau=tau, whole=whole, planes=planes, weights=True, pad=N // 7, seed=K))


@gpu
@pytest.mark.parametrize("N,C,V,K", [(5, 64, 19000, 0), (8, 256, 18944, 3), (7, 4096, 257, 0), (4, 4096, 300, 2), (8, 2080, 1000, 0), (9, 32, 40, 0), (9, 1024, 3001, 4),
                                     (40, 96, 18945, 0), (100, 64, 18977, 5), (128, 160, 25000, 0), (127, 544, 9000, 7), (77, 2048, 3009, 0), (33, 4096, 999, 0)])
@pytest.mark.parametrize("planes", [False, True])
def test_few_and_some_dozens_of_rows(N, C, V, K, planes):
    """Either side of where the kernels change, and shares of W of one to four groups of 32 rows."""
    check(Case(N, C, V, K=K, tau=2.0 if K else 1.0, planes=planes, weights=True, pad=N // 9, seed=N + V))


@gpu
@pytest.mark.parametrize("N", [6, 12, 300])
@pytest.mark.parametrize("K", [0, 9])
def test_gradients_in_pieces_of_the_vocabulary(N, K):
    c = Case(N, 96, 1111, K=K, tau=2.0 if K else 1.0, pad=1)
    lse = c.forward()[1]
    whole = c.backward(lse)
    for piece in (1, 256, 300, 512, 1111, 1 << 30):
        dx, dw, _ = c.backward(lse, piece)
        assert rel(dx, whole[0]) < 2e-6 and rel(dw, whole[1]) < 2e-6
    assert b.bt_op_head_bwd_scratch_bytes(N, 96, 1111, K, 256) <= b.bt_op_head_bwd_scratch_bytes(N, 96, 1111, K, 1024)


@gpu
@pytest.mark.parametrize("N", [5, 50, 200])
def test_outputs_asked_for_one_by_one(N):
    c = Case(N, 64, 700, weights=True, pad=2)
    lse = c.forward()[1]
    dx, dw, ds = c.backward(lse, dx_split=True)
    check_split(ds, dx.cpu().numpy())
    assert torch.equal(c.backward(lse, dw=False)[0], dx)
    assert torch.equal(c.backward(lse, dx=False)[1], dw)
    assert torch.equal(c.backward(lse, dx=False, dw=False, dx_split=True)[2], ds)
    out = torch.full((N,), math.nan, device=DEV)
    work = torch.empty(b.bt_op_head_fwd_scratch_bytes(N, 64, 700), dtype=torch.uint8, device=DEV)
    b.bt_op_head_xent_fwd(c.x, None, c.w, None, c.targets, c.rw, N, 64, 700, c.inv, out, None, None, work, work.numel())
    assert torch.equal(out, c.forward()[0])


@gpu
@pytest.mark.parametrize("N", [5, 40, 200])
def test_planes_of_dx_alone_over_several_pieces(N):
    """The sums over the pieces lie in the hi plane until the last."""
    c = Case(N, 96, 1500, weights=True, pad=1)
    lse = c.forward()[1]
    dx = c.backward(lse, 256)[0]
    ds = c.backward(lse, 256, dx=False, dw=False, dx_split=True)[2]
    check_split(ds, dx.cpu().numpy())
    both = c.backward(lse, 256, dx_split=True)
    assert torch.equal(both[0], dx) and torch.equal(both[2], ds)


@gpu
@pytest.mark.parametrize("N,C,V", [(4, 96, 700), (40, 96, 19000), (40, 1024, 3001), (200, 64, 700)])
@pytest.mark.parametrize("planes", [False, True])
def test_arrays_on_multiples_of_sixteen_bytes(N, C, V, planes):
    """Every array 16 bytes behind a multiple of 256."""
    c = Case(N, C, V, planes=planes, weights=True)
    want = c.forward()
    grads = c.backward(want[1])[:2]
    off = lambda t: None if t is None else torch.cat((torch.zeros(4, device=DEV, dtype=t.dtype), t.reshape(-1)))[4:].view(t.shape)  # noqa: E731
    x, xs, w, ws = (off(t) for t in c.operands())
    targets, rw, lse = off(c.targets), off(c.rw), off(want[1])
    out = [torch.full((n + 4,), math.nan, device=DEV)[4:] for n in (N, N, 1)]
    dx, dw = torch.full((N * C + 4,), math.nan, device=DEV)[4:].view(N, C), torch.full((V * C + 4,), math.nan, device=DEV)[4:].view(V, C)
    work = torch.empty(max(b.bt_op_head_fwd_scratch_bytes(N, C, V), b.bt_op_head_bwd_scratch_bytes(N, C, V)), dtype=torch.uint8, device=DEV)
    b.bt_op_head_xent_fwd(x, xs, w, ws, targets, rw, N, C, V, c.inv, *out, work, work.numel())
    b.bt_op_head_xent_bwd(x, xs, w, ws, targets, rw, lse, N, C, V, c.inv, dx, dw, work, work.numel())
    b.bt_op_head_check(work)
    assert all(torch.equal(p, q) for p, q in zip((*out, dx, dw), (*want, *grads)))


@gpu
@pytest.mark.parametrize("N", [4, 40, 150])
@pytest.mark.parametrize("K", [0, 5])
def test_two_runs_give_the_same_bits(N, K):
    c = Case(N, 160, 3000, K=K, weights=True)
    one, two = c.forward(), c.forward()
    assert all(torch.equal(p, q) for p, q in zip(one, two))
    assert all(torch.equal(p, q) for p, q in zip(c.backward(one[1])[:2], c.backward(one[1])[:2]))


@gpu
@pytest.mark.parametrize("N", [4, 40, 150])
@pytest.mark.parametrize("K", [0, 5])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_rows_without_a_target_may_hold_anything(N, K, value):
    c = Case(N, 64, 900, K=K, pad=2, weights=True)                # row 2 has weight 0
    plain = check(c)
    c.x[:2] = value
    c.x[2, 5] = value
    losses, lse, mean = c.forward()
    assert torch.equal(losses[3:], plain[0][3:]) and torch.equal(lse[3:], plain[1][3:]) and torch.equal(mean, plain[2])
    assert not losses[:2].any()
    dx, dw, _ = c.backward(lse)
    assert torch.equal(dx[3:], plain[3][3:]) and not dx[:3].any() and rel(dw, plain[4]) < 1e-6


@gpu
@pytest.mark.parametrize("N", [4, 40, 150])
def test_a_batch_without_any_target(N):
    for K in (0, 3):
        c = Case(N, 64, 300, K=K, pad=N)
        losses, lse, mean = c.forward()
        assert not losses.any() and float(mean[0]) == 0.0 and torch.isfinite(lse).all()
        dx, dw, _ = c.backward(lse)
        assert not dx.any() and not dw.any()


@gpu
@pytest.mark.parametrize("K", [0, 3])
def test_no_rows(K):
    c = Case(0, 64, 300, K=K)
    assert float(c.forward()[2][0]) == 0.0
    assert not c.backward(torch.empty(0, device=DEV))[1].any()


@gpu
@pytest.mark.parametrize("N", [4, 40, 150])
def test_a_row_that_is_not_a_number_stays_alone(N):
    c = Case(N, 64, 900)
    plain = c.forward()
    c.x[1, 3] = math.nan
    losses, lse, mean = c.forward()
    keep = [i for i in range(N) if i != 1]
    assert torch.isnan(losses[1]) and torch.isnan(lse[1]) and torch.isnan(mean[0])
    assert torch.equal(losses[keep], plain[0][keep]) and torch.equal(lse[keep], plain[1][keep])


@gpu
@pytest.mark.parametrize("N", [5, 40, 150])
def test_ids_behind_the_vocabulary_count_as_zero_and_are_recorded(N):
    c = Case(N, 64, 300)
    c.targets[3] = 300
    bad = torch.zeros(1, dtype=torch.int32, device=DEV)
    losses, lse, _ = c.forward(bad)
    assert int(bad[0]) == 4
    c.targets[3] = 0
    assert torch.equal(losses, c.forward()[0])
    zero = c.backward(lse)
    c.targets[3] = (1 << 31) - 1
    assert all(torch.equal(p, q) for p, q in zip(c.backward(lse)[:2], zero[:2]))
    t = Case(N, 64, 300, K=4)
    t.ids[4, 2] = 300
    bad.zero_()
    losses, lse, _ = t.forward(bad)
    assert int(bad[0]) == 5
    t.ids[4, 2] = 0
    assert torch.equal(losses, t.forward()[0])


@gpu
@pytest.mark.parametrize("N", [4, 50, 200])
@pytest.mark.parametrize("sx,sw", [(1e4, 1e-4), (1e-6, 1e6), (1e-20, 1e20), (1e15, 1e-15), (30.0, 1.0)])
def test_operands_of_any_size(N, sx, sw):
    """The scales cancel in the scores; the last case has scores of some 60, and tolerances relative to them."""
    c = Case(N, 96, 700, seed=3)
    c.x *= sx
    c.w *= sw
    losses, lse, _ = c.forward()
    want = c.want()
    top = float((c.x.double() @ c.w.double().T).abs().max())
    assert float((lse - want[1]).abs().max()) < TOL * max(1.0, top)
    want = c.want(lse)
    dx, dw, _ = c.backward(lse)
    assert rel(dx, want[3]) < TOL * max(1.0, top) and rel(dw, want[4]) < TOL * max(1.0, top)


@gpu
@pytest.mark.parametrize("N", [4, 50, 200])
def test_rows_and_weights_of_unequal_size(N):
    """Rows of x, and their weights in the loss, that differ by 2^20, and columns of W that differ by 2^10: every row of dx is
    right to its own size."""
    c = Case(N, 64, 600, seed=5)
    c.x[1] *= 2.0 ** -20
    c.rw = torch.ones(N, device=DEV)
    c.rw[2] = 2.0 ** -20
    c.w[:, ::2] *= 2.0 ** -10
    lse = c.forward()[1]
    want = c.want(lse)
    dx, dw, _ = c.backward(lse)
    for n in range(N):
        assert rel(dx[n], want[3][n]) < TOL
    assert rel(dw, want[4]) < TOL and rel(dx[:, ::2], want[3][:, ::2]) < TOL


@gpu
@pytest.mark.parametrize("N", [3, 20, 140])
@pytest.mark.parametrize("K", [0, 6])
def test_gradients_against_differences(N, K):
    """dx and dw against central differences of the 64-bit mean loss, along random directions."""
    c = Case(N, 32, 90, K=K, tau=1.5 if K else 1.0, pad=1, weights=True, seed=9)
    lse = c.forward()[1]
    dx, dw, _ = c.backward(lse)
    a, h = c.aims()
    gen = torch.Generator(DEV).manual_seed(1)

    def mean(x, w):
        return head64(x @ w.T / c.tau, a, h, c.tau, c.weight(), c.inv)[2]
    x, w, e = c.x.double(), c.w.double(), 1e-5
    for _ in range(3):
        u, v = torch.randn(x.shape, generator=gen, device=DEV).double(), torch.randn(w.shape, generator=gen, device=DEV).double()
        want = float((mean(x + e * u, w + e * v) - mean(x - e * u, w - e * v)) / (2 * e))
        size = float((dx.double() ** 2 * u ** 2).sum().sqrt() + (dw.double() ** 2 * v ** 2).sum().sqrt())
        # e^2 / 6 times a third derivative of order one is 2e-11; lse is an FP32 value, 2^-24 of some units
        assert abs(float((dx.double() * u).sum() + (dw.double() * v).sum()) - want) < 2 * TOL * size


@gpu
def test_far_rows_and_vocabulary():
    """Offsets past 2^31 elements: W of 2^24 / 8 rows of 1,056 columns (2.2e9 values)."""
    V, C, N = (1 << 24) // 8, 1056, 3
    gen = torch.Generator(DEV).manual_seed(2)
    w = torch.randn(V, C, generator=gen, device=DEV) * 0.03
    x = torch.randn(N, C, generator=gen, device=DEV)
    t = torch.tensor([V - 1, 5, V // 2], dtype=torch.int32, device=DEV)
    for n in (N, 20):
        xs = x.repeat(8, 1)[:n].contiguous()
        ts = t.repeat(8)[:n].contiguous()
        losses, lse, mean = (torch.empty(k, device=DEV) for k in (n, n, 1))
        work = torch.empty(b.bt_op_head_fwd_scratch_bytes(n, C, V), dtype=torch.uint8, device=DEV)
        b.bt_op_head_xent_fwd(xs, None, w, None, ts, None, n, C, V, 1.0 / n, losses, lse, mean, work, work.numel())
        b.bt_op_head_check(work)
        z = torch.cat([xs.double() @ w[i:i + V // 16].double().T for i in range(0, V, V // 16)], 1)
        want = torch.logsumexp(z, 1)
        assert float((lse - want).abs().max()) < TOL * 10
        assert float((losses - (want - z.gather(1, ts.long()[:, None])[:, 0])).abs().max()) < TOL * 10
        dw = torch.empty_like(w)
        dx = torch.empty_like(xs)
        work = torch.empty(b.bt_op_head_bwd_scratch_bytes(n, C, V), dtype=torch.uint8, device=DEV)
        b.bt_op_head_xent_bwd(xs, None, w, None, ts, None, lse, n, C, V, 1.0 / n, dx, dw, work, work.numel())
        b.bt_op_head_check(work)
        d = torch.exp(z - lse.double()[:, None])
        d[torch.arange(n, device=DEV), ts.long()] -= 1.0
        d /= n
        for v in (0, 5, V // 2, V - 1):
            assert rel(dw[v], d[:, v] @ xs.double()) < 1e-4        # rows of single columns: relative to small sums
        want = sum(d[:, i:i + V // 16] @ w[i:i + V // 16].double() for i in range(0, V, V // 16))
        assert rel(dx, want) < TOL
        del work, dw, z, d


@gpu
@pytest.mark.parametrize("N", [4, 40, 150])
def test_captured_calls_and_another_stream(N):
    c = Case(N, 64, 500, weights=True)
    plain = check(c)
    out = [torch.empty(n, device=DEV) for n in (N, N, 1)]
    dx, dw = torch.empty(N, 64, device=DEV), torch.empty(500, 64, device=DEV)
    fs = torch.empty(b.bt_op_head_fwd_scratch_bytes(N, 64, 500), dtype=torch.uint8, device=DEV)
    bs = torch.empty(b.bt_op_head_bwd_scratch_bytes(N, 64, 500), dtype=torch.uint8, device=DEV)

    def step():
        b.bt_op_head_xent_fwd(c.x, None, c.w, None, c.targets, c.rw, N, 64, 500, c.inv, *out, fs, fs.numel())
        b.bt_op_head_xent_bwd(c.x, None, c.w, None, c.targets, c.rw, out[1], N, 64, 500, c.inv, dx, dw, bs, bs.numel())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip((*out, dx, dw), plain))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x = c.x.clone()
    c.x.copy_(x.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip((*out, dx, dw), check(c)))
    c.x.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip((*out, dx, dw), plain))


@gpu
def test_rows_behind_the_last_are_left_alone():
    for N in (3, 30, 130):
        c = Case(N, 64, 200)
        big = torch.full((N + 40, 64), 7.0, device=DEV)
        lse = c.forward()[1]
        losses = torch.full((N + 40,), 7.0, device=DEV)
        work = torch.empty(b.bt_op_head_bwd_scratch_bytes(N, 64, 200), dtype=torch.uint8, device=DEV)
        dw = torch.full((260, 64), 7.0, device=DEV)
        b.bt_op_head_xent_bwd(c.x, None, c.w, None, c.targets, None, lse, N, 64, 200, c.inv, big, dw, work, work.numel())
        work = torch.empty(b.bt_op_head_fwd_scratch_bytes(N, 64, 200), dtype=torch.uint8, device=DEV)
        b.bt_op_head_xent_fwd(c.x, None, c.w, None, c.targets, None, N, 64, 200, c.inv, losses, None, None, work, work.numel())
        torch.cuda.synchronize()
        assert (big[N:] == 7).all() and (dw[200:] == 7).all() and (losses[N:] == 7).all()
        assert not (big[:N] == 7).any() and not (dw[:200] == 7).any()


@gpu
def test_scratch_is_enough_and_not_exceeded():
    for N, C, V, K in ((3, 64, 100, 5), (12, 64, 300, 3), (60, 96, 700, 4), (150, 96, 700, 0), (300, 64, 5000, 9)):
        c = Case(N, C, V, K=K)
        lse = c.forward()[1]
        for back in (False, True):
            need = (b.bt_op_head_bwd_scratch_bytes if back else b.bt_op_head_fwd_scratch_bytes)(N, C, V, K)
            area = torch.full((need + 4096,), 90, dtype=torch.uint8, device=DEV)
            if back:
                call = b.bt_op_head_distill_bwd if K else b.bt_op_head_xent_bwd
                call(c.x, None, c.w, None, c.aim(), None, lse, N, C, V, c.inv, torch.empty(N, C, device=DEV),
                     torch.empty(V, C, device=DEV), area, need)
            else:
                c.forward(scratch=area)
            torch.cuda.synchronize()
            assert (area[need:] == 90).all()


@gpu
@pytest.mark.parametrize("N", [6, 40, 150])
@pytest.mark.parametrize("K,V", [(20, 7), (32, 40), (33, 9), (64, 3000), (100, 11), (300, 200), (1024, 37), (1024, 3000)])
def test_an_id_many_times(N, K, V):
    """Entries of one id, next to one another, far apart and in every place, and ids in even steps."""
    c = Case(N, 32, V, K=K, tau=2.0, seed=K + V)
    k = torch.arange(K, device=DEV)
    c.ids[1] = 3                                                  # all of them
    c.ids[2] = (k % V).int()
    c.ids[3] = (64 * k % V).int()
    c.ids[4] = (k * 8 // K % V).int()
    c.ids[5] = -1
    c.ids[5, 0] = c.ids[5, K - 1] = V - 1                         # the first and the last
    check(c)


@gpu
@pytest.mark.parametrize("N", [4, 40, 150])
@pytest.mark.parametrize("K", [5, 40])
def test_captured_distillation(N, K):
    c = Case(N, 64, 500, K=K, tau=1.5, weights=True)
    plain = check(c)
    out = [torch.empty(n, device=DEV) for n in (N, N, 1)]
    dx, dw = torch.empty(N, 64, device=DEV), torch.empty(500, 64, device=DEV)
    fs = torch.empty(b.bt_op_head_fwd_scratch_bytes(N, 64, 500, K), dtype=torch.uint8, device=DEV)
    bs = torch.empty(b.bt_op_head_bwd_scratch_bytes(N, 64, 500, K), dtype=torch.uint8, device=DEV)
    aim = c.aim()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.bt_op_head_distill_fwd(c.x, None, c.w, None, aim, c.rw, N, 64, 500, c.inv, *out, fs, fs.numel())
        b.bt_op_head_distill_bwd(c.x, None, c.w, None, aim, c.rw, out[1], N, 64, 500, c.inv, dx, dw, bs, bs.numel())
    ids = c.ids.clone()
    c.ids.copy_((ids + 7) % 500)                                  # the table of the last run's entries must not stay
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip((*out, dx, dw), check(c)))
    c.ids.copy_(ids)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip((*out, dx, dw), plain))


@gpu
@pytest.mark.parametrize("N", [4, 40, 300])
def test_two_calls_at_once(N):
    """Two calls with a scratch each, on two streams."""
    cases = [Case(N, 128, 9000, weights=True, seed=1), Case(N, 128, 9000, K=12, weights=True, seed=2)]
    plain = [check(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                call_f, call_b = (b.bt_op_head_distill_fwd, b.bt_op_head_distill_bwd) if c.K else (b.bt_op_head_xent_fwd, b.bt_op_head_xent_bwd)
                out = [torch.empty(n, device=DEV) for n in (N, N, 1)] + [torch.empty(N, 128, device=DEV), torch.empty(9000, 128, device=DEV)]
                need = max(b.bt_op_head_fwd_scratch_bytes(N, 128, 9000, c.K), b.bt_op_head_bwd_scratch_bytes(N, 128, 9000, c.K))
                work = torch.empty(need, dtype=torch.uint8, device=DEV)
                aim = c.aim()
                call_f(c.x, None, c.w, None, aim, c.rw, N, 128, 9000, c.inv, *out[:3], work, need)
                call_b(c.x, None, c.w, None, aim, c.rw, out[1], N, 128, 9000, c.inv, *out[3:], work, need)
                got.append((out, work, aim))
        torch.cuda.synchronize()
        for (out, _, _), want in zip(got, plain):
            assert all(torch.equal(p, q) for p, q in zip(out, want))


@gpu
def test_no_rows_leave_no_error():
    work = torch.full((4096,), 255, dtype=torch.uint8, device=DEV)
    none, w, dw, mean = torch.empty(0, device=DEV), torch.ones(8, 32, device=DEV), torch.ones(8, 32, device=DEV), torch.ones(1, device=DEV)
    b.bt_op_head_xent_fwd(None, None, w, None, None, None, 0, 32, 8, 1.0, None, None, mean, work, 4096)
    b.bt_op_head_check(work)
    work.fill_(255)
    b.bt_op_head_xent_bwd(None, None, w, None, None, None, none, 0, 32, 8, 1.0, None, dw, work, 4096)
    b.bt_op_head_check(work)
    assert float(mean) == 0.0 and not dw.any()


# ------------------------------------------------------------------------------- GPU: distillation on logits

def logits_case(N, V, K, tau, whole, pad, seed=0, ld=None):
    c = Case(N, 32, V, K=K, tau=tau, whole=whole, weights=True, pad=pad, seed=seed)
    ld = ld or (V + 3) // 4 * 4
    c.z = torch.randn(N, ld, generator=torch.Generator(DEV).manual_seed(seed), device=DEV) * 3
    c.ld = ld
    return c


def logits_want(c):
    losses, own, mean, d = head64(c.z[:, :c.V].double() / c.tau, *c.aims(), c.tau, c.weight(), c.inv)
    full = torch.zeros(c.N, c.ld, dtype=torch.float64, device=DEV)
    full[:, :c.V] = d
    return losses, mean, full


def logits_run(c, dz=True, planes=False, z=None, over=None, bad=None):
    losses, mean = torch.full((c.N,), math.nan, device=DEV), torch.full((1,), math.nan, device=DEV)
    g = torch.full((c.N, c.ld), math.nan, device=DEV) if dz else None
    s = torch.full((2, c.N, c.ld), math.nan, device=DEV) if planes else None
    z = c.z if z is None else z
    b.bt_op_softmax_distill(z, c.aim(), c.rw, c.N, c.V, c.ld, c.inv, losses, mean, over if over is not None else g, s, bad)
    return losses, mean, g, s


@gpu
@pytest.mark.parametrize("N,V,K,tau,whole,ld", [(1, 1, 1, 1.0, False, 4), (1, 50304, 16, 2.0, False, None), (3, 5, 8, 0.5, True, 12), (7, 513, 64, 1.0, True, 520),
                                                (300, 511, 3, 2.0, False, None), (700, 2050, 33, 1.5, True, 2304), (150, 8193, 100, 1.0, False, None),
                                                (400, 24577, 5, 4.0, False, None), (161, 50257, 64, 2.0, True, 50304), (620, 51200, 9, 1.0, False, None),
                                                (20, 51201, 12, 1.0, False, None), (12, 131071, 1024, 2.0, True, 131072), (5, 262147, 30, 1.0, False, None),
                                                (2, 700001, 30, 1.0, True, None)])
def test_distillation_on_logits(N, V, K, tau, whole, ld):
    c = logits_case(N, V, K, tau, whole, pad=N // 6, seed=V, ld=ld)
    losses, mean, g, s = logits_run(c, planes=True)
    want = logits_want(c)
    # FP32 sums and exponentials of scores of some units: a few 2^-24 of them
    top = max(1.0, float(c.z.abs().max()) / tau)
    assert float((losses - want[0]).abs().max()) < 2e-6 * tau ** 2 * top * (float(c.aims()[0].sum(1).max()) + 1)
    assert abs(float(mean[0]) - float(want[1])) < 4e-6 * tau ** 2 * top
    assert rel(g, want[2]) < 2e-6 * top and not g[:, V:].any() and not g[want[2].abs().sum(1) == 0].any()
    check_split(s, g.cpu().numpy())
    alone = logits_run(c, dz=False)
    assert torch.equal(alone[0], losses) and torch.equal(alone[1], mean)
    assert torch.equal(logits_run(c, dz=False, planes=True)[3], s)


@gpu
@pytest.mark.parametrize("N", [6, 300])
@pytest.mark.parametrize("K,V", [(20, 7), (32, 40), (33, 9), (64, 3000), (300, 9000), (1024, 37), (1024, 24577), (512, 100001)])
def test_an_id_many_times_on_logits(N, K, V):
    c = logits_case(N, V, K, 2.0, False, pad=0, seed=K + V)
    k = torch.arange(K, device=DEV)
    c.ids[1] = 3
    c.ids[2] = (k % V).int()
    c.ids[3] = (64 * k % V).int()
    c.ids[4] = (k * 8 // K % V).int()
    c.ids[5] = -1
    c.ids[5, 0] = c.ids[5, K - 1] = V - 1
    losses, _, g, _ = logits_run(c)
    want = logits_want(c)
    top = max(1.0, float(c.z.abs().max()) / 2)                    # as above
    assert float((losses - want[0]).abs().max()) < 2e-6 * 4 * top * 2
    assert rel(g, want[2]) < 2e-6 * top


@gpu
@pytest.mark.parametrize("N,V", [(3, 900), (640, 50257), (4, 60001)])
def test_gradient_over_the_logits(N, V):
    c = logits_case(N, V, 20, 1.5, False, pad=1, ld=(V + 67) // 4 * 4)
    losses, mean, g, s = logits_run(c, planes=True)
    z = c.z.clone()
    got = logits_run(c, z=z, over=z)
    assert torch.equal(got[0], losses) and torch.equal(z, g)
    both = torch.empty(2, N, c.ld, device=DEV)
    both[0].copy_(c.z)
    l2, m2 = torch.empty(N, device=DEV), torch.empty(1, device=DEV)
    b.bt_op_softmax_distill(both[0], c.aim(), c.rw, N, V, c.ld, c.inv, l2, m2, None, both)
    assert torch.equal(both, s) and torch.equal(l2, losses) and torch.equal(m2, mean)


@gpu
def test_logits_of_rows_without_entries_and_behind_the_vocabulary_may_hold_anything():
    c = logits_case(40, 700, 6, 1.0, False, pad=3, ld=712)
    plain = logits_run(c)
    c.z[:, 700:] = math.nan
    c.z[0], c.z[1], c.z[2, 9] = math.nan, math.inf, -math.inf
    got = logits_run(c)
    for p, q in zip(got[:3], plain[:3]):
        assert torch.equal(p, q)


@gpu
def test_logits_of_minus_infinity():
    """Columns that the student rules out: probability and gradient zero; a row of the teacher's that wants one has infinite loss."""
    c = logits_case(30, 300, 4, 1.0, False, pad=0)
    c.ids[:] = torch.arange(4, dtype=torch.int32, device=DEV) * 50
    c.top[c.top == -math.inf] = 0.5
    c.z[:, 10:20] = -math.inf
    c.z[5] = torch.finfo(torch.float32).min
    losses, mean, g, _ = logits_run(c)
    want = logits_want(c)
    keep = [i for i in range(30) if i != 5]
    assert rel(g[keep], want[2][keep]) < 2e-5 and not g[:, 10:20][keep].any()
    assert float((losses[keep] - want[0][keep]).abs().max()) < 2e-5
    assert torch.isfinite(g[5]).all() and rel(g[5], want[2][5]) < 2e-5     # a constant row is a uniform one
    c.ids[3, 1] = 12
    assert math.isinf(float(logits_run(c)[0][3]))


@gpu
def test_ids_behind_the_vocabulary_on_logits():
    c = logits_case(30, 300, 4, 1.0, False, pad=0)
    c.ids[7, 1] = 300
    bad = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = logits_run(c, bad=bad)
    assert int(bad[0]) == 8
    c.ids[7, 1] = 0
    assert all(torch.equal(p, q) for p, q in zip(got[:3], logits_run(c)[:3]))


@gpu
def test_no_rows_of_logits():
    c = Case(0, 32, 300, K=4)
    mean = torch.full((1,), 3.0, device=DEV)
    b.bt_op_softmax_distill(torch.empty(0, 300, device=DEV), c.aim(), None, 0, 300, 300, 1.0, torch.empty(0, device=DEV), mean, None)
    assert float(mean[0]) == 0.0


# ------------------------------------------------------------------------------- GPU: together, and beside the training step

@gpu
@pytest.mark.parametrize("N", [6, 77, 333])
def test_hard_and_soft_loss_of_a_student(N):
    """0.3 cross entropy + 0.7 distillation on the same rows, from hidden states and from logits made by the library's GEMM,
    against 64-bit automatic differentiation of the sum."""
    C, V, K, tau = 96, 1024, 12, 2.0
    hard, soft = Case(N, C, V, pad=2, seed=1), Case(N, C, V, K=K, tau=tau, pad=1, seed=1)
    hard.inv, soft.inv = 0.3 / N, 0.7 / N
    lh, eh, mh = hard.forward()
    ls, es, ms = soft.forward()
    dx = hard.backward(eh)[0] + soft.backward(es)[0]
    dw = hard.backward(eh)[1] + soft.backward(es)[1]

    x, w = hard.x.double().requires_grad_(), hard.w.double().requires_grad_()
    z = x @ w.T
    t = hard.targets.long()
    ce = torch.nn.functional.cross_entropy(z, t, ignore_index=-1, reduction="none")
    a, h = soft.aims()
    kd = tau ** 2 * (h - (a * torch.log_softmax(z / tau, 1)).sum(1))
    total = (0.3 * ce.sum() + 0.7 * kd.sum()) / N
    total.backward()
    assert abs(float(mh[0] + ms[0]) - float(total.detach())) < TOL * 20
    assert rel(dx, x.grad) < TOL and rel(dw, w.grad) < TOL

    M = (N + 3) // 4 * 4
    xs = torch.zeros(M, C, device=DEV)
    xs[:N] = hard.x
    out = torch.empty(M, V, device=DEV)
    nb = b.bt_op_gemm_scratch_bytes(b.BT_GEMM_NT, M, V, C)
    b.bt_op_gemm(b.BT_GEMM_NT, M, V, C, xs, hard.w, out, None, None, torch.empty(nb, dtype=torch.uint8, device=DEV), nb)
    logits = out[:N].contiguous()
    soft.z, soft.ld = logits, V
    l2, m2, g, _ = logits_run(soft)
    assert float((l2 - ls).abs().max()) < TOL * 20 and rel(g.double() @ hard.w.double(), soft.want(es)[3]) < 2 * TOL


@gpu
def test_head_loss_of_a_model():
    """Loss and gradients of the head from a model's own last hidden states and tied weights: the loss is the model's, dw the
    part of the tied gradient that comes from the head."""
    import seeded_inputs as si
    cfg = si.config(0)
    m = b.Model(cfg["n_layers"], cfg["d_model"], cfg["n_heads"], cfg["seq_len"], cfg["vocab_size"], cfg["padded_vocab_size"], cfg["batch"])
    m.load_params(si.init_params(cfg, 0))
    tok, tgt = si.tokens_for(cfg, 0)
    tok, tgt = torch.as_tensor(tok).to(DEV), torch.as_tensor(tgt).to(DEV)
    loss = m.forward(tok, tgt)
    N, C, V = tok.numel(), cfg["d_model"], cfg["padded_vocab_size"]
    xf = m.activation("xf", planes=2).view(2, N, C)
    w = m.tensor("wte").view(V, C)
    t = tgt.reshape(-1).int().contiguous()
    losses, lse, mean = (torch.empty(n, device=DEV) for n in (N, N, 1))
    work = torch.empty(b.bt_op_head_fwd_scratch_bytes(N, C, V), dtype=torch.uint8, device=DEV)
    b.bt_op_head_xent_fwd(None, xf, w, None, t, None, N, C, V, 1.0 / N, losses, lse, mean, work, work.numel())
    assert abs(float(mean[0]) - loss) < 1e-5 * loss
    assert rel(losses, m.activation("losses")) < 1e-5
    dlogits = m.activation("dlogits", planes=2).view(2, N, V).double().sum(0)
    dx, dw = torch.empty(N, C, device=DEV), torch.empty(V, C, device=DEV)
    work = torch.empty(b.bt_op_head_bwd_scratch_bytes(N, C, V), dtype=torch.uint8, device=DEV)
    b.bt_op_head_xent_bwd(None, xf, w, None, t, None, lse, N, C, V, 1.0 / N, dx, dw, work, work.numel())
    assert rel(dx, dlogits @ w.double()) < TOL and rel(dw, dlogits.T @ xf.double().sum(0)) < TOL
    m.close()
