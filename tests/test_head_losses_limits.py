"""The losses at the language-model head, and distillation on logits, where they could give way: teachers whose numbers are not
finite beside entries that are not there; rows of which most CTAs have nothing; rows that are sure of their target; words
that are improbable everywhere."""
import math

import pytest
import torch

from paper_2606_24780_b200 import binding as b

from gpu_util import DEV
from test_head_losses import TOL, Case, lib, logits_case, logits_run, logits_want, refused  # noqa: F401

gpu = pytest.mark.gpu


# ------------------------------------------------------------------------------- CPU: scratch

def test_a_piece_of_the_vocabulary_is_a_multiple_of_256_columns(lib):
    """Sizes of the scratch for pieces asked for, and for the library's own."""
    C, V = 32, 50000
    for N in (9, 300, 1 << 20, 1 << 24):
        size = lambda piece: b.bt_op_head_bwd_scratch_bytes(N, C, V, 0, piece)  # noqa: E731
        rest = size(256) - 1024 * N
        assert size(1) == size(255) == size(256) and size(257) == size(512)
        for piece in (256, 512, 1000, 50000, 1 << 30):
            pieces = -(-V // min(-(-piece // 256) * 256, 1 << 30))
            assert size(piece) == rest + 4 * N * (-(-(-(-V // pieces)) // 256) * 256)
        own = -(-max(256, (1 << 27) // N) // 256) * 256
        assert size(0) == size(own) and size(0) - rest <= max(4 * N * 256, (1 << 29) + 4 * N * 256)


def test_losses_over_the_logits_and_dlogits_over_its_planes_are_refused(lib):
    P, N, ld = 0x10000, 4, 100
    z, lo = 5 * P, 4 * N * ld

    def call(losses=2 * P, mean=None, dz=None, planes=None):
        b.bt_op_softmax_distill(z, b.bt_distill(4, 1.0, P, P, None), None, N, ld, ld, 1.0, losses, mean, dz, planes, None, 0)

    for bad in (dict(losses=z), dict(mean=z), dict(dz=6 * P, planes=6 * P), dict(dz=6 * P + lo, planes=6 * P), dict(dz=z, planes=z)):
        refused(lambda: call(**bad))


# ------------------------------------------------------------------------------- GPU: teachers that are not finite

def spoil(c, kind, row):
    """A row whose teacher has no finite normaliser, between entries that are not there (far below zero, and by a logit of -inf)."""
    c.ids[row, 1], c.ids[row, 3] = -100, -(1 << 31)
    c.top[row, 0] = 1.0
    c.top[row, 4] = -math.inf
    if kind.startswith("lse"):
        c.top_lse[row] = float(kind[4:])
    else:
        c.top[row, 2] = {"nan": math.nan, "inf": math.inf, "overflow": torch.finfo(torch.float32).max}[kind]


@gpu
@pytest.mark.parametrize("N", [4, 40, 150])
@pytest.mark.parametrize("kind", ["nan", "inf", "overflow", "lse nan", "lse -inf"])
def test_a_teacher_that_is_not_finite_stays_in_its_row(N, kind):
    """"overflow": the logit is finite and leaves FP32 when it is divided by the temperature."""
    make = lambda: Case(N, 64, 900, K=6, tau=0.5, whole=kind.startswith("lse"), weights=True)  # noqa: E731
    c, plain = make(), make()
    # a row of weight 1, whose other entries are whole in both
    row = 3
    for k in (c, plain):
        k.ids[row] = torch.arange(6, dtype=torch.int32, device=DEV) * 7
    spoil(c, kind, row)
    want, got = plain.forward(), c.forward()
    keep = [i for i in range(N) if i != row]
    assert not torch.isfinite(got[0][row]) and not torch.isfinite(got[2][0])
    assert torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[1], want[1])
    dx = c.backward(got[1], dw=False)[0]
    assert not torch.isfinite(dx[row]).any() and torch.equal(dx[keep], plain.backward(want[1], dw=False)[0][keep])


@gpu
@pytest.mark.parametrize("N,V", [(6, 900), (300, 900), (6, 50257)])
@pytest.mark.parametrize("kind", ["nan", "inf", "overflow", "lse nan", "lse -inf"])
def test_a_teacher_that_is_not_finite_stays_in_its_row_of_logits(N, V, kind):
    make = lambda: logits_case(N, V, 6, 0.5, kind.startswith("lse"), pad=0)  # noqa: E731
    c, plain = make(), make()
    row = 3
    for k in (c, plain):
        k.ids[row] = torch.arange(6, dtype=torch.int32, device=DEV) * 7
    spoil(c, kind, row)
    want, got = logits_run(plain), logits_run(c)
    keep = [i for i in range(N) if i != row]
    assert not torch.isfinite(got[0][row]) and not torch.isfinite(got[1][0])
    assert torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[2][keep], want[2][keep])


# ------------------------------------------------------------------------------- GPU: slices of a row on a cluster

@gpu
@pytest.mark.parametrize("N,V,ld", [(1, 5, 20000), (30, 3, 20480), (37, 2500, 40004), (74, 1, 8300), (148, 9, 16400), (3, 16390, 17000), (2, 1, 1 << 20)])
def test_rows_whose_vocabulary_ends_in_the_first_slices(N, V, ld):
    """CTAs of a cluster that have no column to read are done with their part of the row long before the others: clusters of
    two, four and eight, several times over."""
    c = logits_case(N, V, 5, 1.5, False, pad=N // 6, seed=ld, ld=ld)
    c.z[:, V:] = math.nan
    losses, mean, d = logits_want(c)
    top = max(1.0, float(c.z[:, :V].abs().max()) / 1.5)           # as test_distillation_on_logits
    for _ in range(5):
        got = logits_run(c)
        assert float((got[0] - losses).abs().max()) < 2e-6 * 1.5 ** 2 * top * 2
        assert abs(float(got[1][0]) - float(mean)) < 4e-6 * 1.5 ** 2 * top
        assert float((got[2] - d).norm()) < 2e-6 * top * c.inv * 1.5 * 2 * float(c.weight().norm()) and not got[2][:, V:].any()


# ------------------------------------------------------------------------------- GPU: rows that are sure of their target

def sure(c, y, top, kind):
    """Scores of `top` at column y of every row, by operands whose products all have one sign or are one product alone."""
    if kind == "aligned":
        c.w[y] = c.x * (top / (c.x.double() ** 2).sum(1, keepdim=True)).float()
    else:
        c.x.zero_()
        c.w[:, 0] = 0
        c.x[:, 0] = 1.0
        c.w[y, 0] = top
    # the products' bound: two operands of 2^-23, the product of their low halves, 72 instructions cut by up to 2^-23 of the running
    # sum, and what is put back for that (2^-24 for each of them)
    return (72 * 2.0 ** -23 + 72 * 2.0 ** -24 + 2.0 ** -21) * float((c.x.abs() @ c.w.abs().T).max())


@gpu
@pytest.mark.parametrize("N,C,V", [(1, 768, 50257), (2, 4096, 300), (4, 96, 9001), (6, 768, 20000), (8, 2080, 999), (40, 768, 19000), (100, 64, 5001), (128, 1056, 700),
                                   (129, 768, 2000), (300, 768, 5003), (1025, 96, 1500)])
@pytest.mark.parametrize("kind", ["aligned", "alone"])
@pytest.mark.parametrize("top", [9.0, 30.0, 70.0])
@pytest.mark.parametrize("planes", [False, True])
def test_the_loss_of_a_row_that_is_sure_of_its_target(N, C, V, kind, top, planes):
    """The loss is log sum_v exp(z_v - z_y): score errors e move it by (1 - q_y) times their differences, however large the scores
    are, and it is not below zero.  The exponentials of a sum, its logarithm and what they are rounded by come to 2^-21."""
    c = Case(N, C, V, planes=planes, seed=N + C, scale=0.5)
    y = torch.arange(N, device=DEV) * 7 % V
    c.targets = y.int()
    e = sure(c, y, top, kind)
    losses, lse, mean = c.forward()
    want = c.want()
    other = 1.0 - torch.exp(-want[0])
    assert (losses >= 0).all()
    assert ((losses.double() - want[0]).abs() <= 2 * e * other + 2.0 ** -21 + 2.0 ** -22 * want[0]).all()
    assert abs(float(mean[0]) - float(want[2])) <= 2 * e * float(other.max()) + 2.0 ** -20 + 2.0 ** -22 * float(want[2])
    assert float((lse - want[1]).abs().max()) <= e + 2.0 ** -21 + 2.0 ** -23 * float(want[1].abs().max())


@gpu
@pytest.mark.parametrize("N,C,V,K", [(1, 768, 50257, 5), (4, 96, 9001, 40), (7, 2080, 999, 3), (9, 64, 40, 33), (40, 768, 19000, 8), (100, 64, 5001, 300), (128, 1056, 700, 64),
                                     (77, 96, 40001, 1), (129, 768, 2000, 33), (1025, 96, 1500, 6)])
@pytest.mark.parametrize("top", [9.0, 30.0, 70.0])
@pytest.mark.parametrize("tau,whole", [(1.0, False), (2.0, True)])
@pytest.mark.parametrize("planes", [False, True])
def test_the_loss_of_a_student_as_sure_as_its_teacher(N, C, V, K, top, tau, whole, planes):
    """An entry's part is p (l + d): l = log p is the logit's distance from the largest one, or from lse, d the distance of log sum exp from
    the score.  Score errors e move d by 2 e (1 - q); it is rounded by 2^-21 and 2^-22 of itself.  l is off by two roundings of what it is
    formed from, and by the exponentials in its sum; p by the same and 2^-22; the sum over the entries by 2^-20 of its parts."""
    c = Case(N, C, V, K=K, tau=tau, planes=planes, seed=N + C, scale=0.5)
    y = torch.arange(N, device=DEV) * 7 % V
    e = sure(c, y, top, "aligned") / tau
    c.ids[:, 0] = y.int()
    c.top = c.top.clamp(-9.0, 9.0)
    c.top[:, 0] = top
    if whole:
        c.top_lse = (torch.logsumexp(c.top.double() / tau, 1) + 0.01).float()
    losses, lse, _ = c.forward()
    want = c.want()
    t = c.top.double() / tau
    log_p = t - (c.top_lse.double() if whole else torch.logsumexp(t, 1))[:, None]
    d = want[1][:, None] - (c.x.double() @ c.w.double().T / tau).gather(1, c.ids.long())
    off = 2.0 ** -22 + 2.0 ** -23 * ((0.0 if whole else t.max(1, keepdim=True)[0] - t) + log_p.abs())
    part = 2 * e * (1.0 - torch.exp(-d)) + 2.0 ** -21 + 2.0 ** -22 * d + off + (off + 2.0 ** -20) * (log_p + d).abs()
    assert ((losses.double() - want[0]).abs() <= tau ** 2 * (torch.exp(log_p) * part).sum(1)).all()
    assert float((lse - want[1]).abs().max()) <= e + 2.0 ** -21 + 2.0 ** -23 * float(want[1].abs().max())


# ------------------------------------------------------------------------------- GPU: improbable words

@gpu
@pytest.mark.parametrize("N", [4, 8, 40, 128, 150, 600])
@pytest.mark.parametrize("K", [0, 3])
@pytest.mark.parametrize("planes", [False, True])
def test_gradients_of_improbable_words_row_by_row(N, K, planes):
    """Words that every row gives a probability of some 2^-20, 2^-30 and 2^-42.  q is held to 2^-40 from nine rows on, and to its own
    size in plain FP32.  A score error e moves q by e q; weights, sums of up to 72 products cut by 2^-23 each and roundings
    come to 2^-16 of the sum of the parts; g_n x_n is held to 2^-40 of the largest."""
    C, V = 768, 900
    c = Case(N, C, V, K=K, planes=planes, seed=N + K, scale=0.25)
    c.x[:, 0] = 4.0
    bits = torch.zeros(V, device=DEV)
    bits[100:200], bits[200:300], bits[300:400] = 10.0, 20.0, 32.0            # beside the 2^-10 of one word of 900
    c.w[:, 0] = -bits * math.log(2.0) / 4.0
    (c.ids if K else c.targets).remainder_(100)                               # aims elsewhere
    lse = c.forward()[1]
    want = c.want(lse)[4]
    _, dw, _ = c.backward(lse, dx=False)
    q = torch.exp(c.x.double() @ c.w.double().T - lse.double()[:, None])
    e = (72 * 2.0 ** -23 + 72 * 2.0 ** -24 + 2.0 ** -21) * float((c.x.abs() @ c.w.abs().T).max())
    size = c.x.double().norm(dim=1) * c.inv
    held = 0.0 if N <= 8 else 2.0 ** -40
    bound = (size[:, None] * (held + (e + 2.0 ** -16) * q + 2.0 ** -40 * math.sqrt(C) * q)).sum(0)
    part = slice(100, 400)                                                    # no aims: sums of parts of one sign in q
    assert ((dw.double() - want).norm(dim=1)[part] <= bound[part]).all()
    assert float(q[:, 100:200].max()) < 2.0 ** -17 and float(q[:, 300:400].max()) < 2.0 ** -39


# ------------------------------------------------------------------------------- GPU: what the tensor core cuts

CUT = 0.28 * 2.0 ** -24         # what is put back per instruction


def instructions(N):
    """Between two sums in registers, C a multiple of 384: three for 16 of the contraction index, of 64 or of 384."""
    return 12 if N <= 128 else 72


@gpu
@pytest.mark.parametrize("N", [128, 2000])
@pytest.mark.parametrize("planes", [False, True])
def test_what_is_put_back_for_cut_sums_is_their_mean(N, planes):
    """Random operands, for which it is measured: within a quarter of it on the mean over all rows, and the 2^-23 by which constants
    (log2 e, ln 2, their product with what is put back) are rounded; without it, or with twice as much, the test fails.  lse is the
    largest score, of some 50, and little more; single scores are off by the products' bound."""
    c = Case(N, 1152, 3000, planes=planes, seed=N, scale=16.0)
    lse, want = c.forward()[1], c.want()[1]
    off = (lse.double() - want) / want
    assert abs(float(off.mean())) < CUT * instructions(N) / 4 + 2.0 ** -23
    bound = (instructions(N) * 2.0 ** -23 + CUT * instructions(N) + 2.0 ** -21) * float((c.x.abs() @ c.w.abs().T).max())
    assert float((lse - want).abs().max()) < bound


@gpu
@pytest.mark.parametrize("N", [128, 2000])
@pytest.mark.parametrize("planes", [False, True])
def test_scores_of_one_product_get_what_is_put_back_and_no_more(N, planes):
    """One number in every row of x and of W, both FP16 ones: nothing is cut, and lse is too large by what is put back; constants are
    rounded by 2^-23, and a score, a sum and a product by 2^-24 each."""
    c = Case(N, 1152, 1500, planes=planes, seed=N)
    c.x.zero_()
    c.w.zero_()
    c.x[:, 700] = 1.5
    c.w[::3, 700] = 20.0
    lse, want = c.forward()[1], c.want()[1]
    off = (lse.double() - want) / 30.0                            # the sum's logarithm, 6.2, has no part in it
    own = 5 * 2.0 ** -24 * 36.2 / 30.0
    assert (off > CUT * instructions(N) - own).all() and (off < CUT * instructions(N) + own).all()


@gpu
@pytest.mark.parametrize("N", [128, 2000])
@pytest.mark.parametrize("C", [384, 1152, 3456])
def test_sums_of_products_of_one_sign(N, C):
    """A sum that grows evenly over n instructions, cut by up to 2^-23 of what it is at each: by 2^-24 n at most over all, less what is put
    back.  Both bounds with the operands' 2^-22 and lse's own 2^-22."""
    c = Case(N, C, 900, seed=C)
    c.x, c.w = c.x.abs() + 0.5, c.w.abs() * 0.1
    c.w[::3] = c.w[::3].sign().abs() + 0.5 * c.w[::3]
    c.w *= 40.0 / float((c.x @ c.w.T).max())
    lse, want = c.forward()[1], c.want()[1]
    off = (lse.double() - want) / want
    n = instructions(N)
    assert (off > -(2.0 ** -24 - CUT) * n - 2.0 ** -21).all() and (off < CUT * n + 2.0 ** -21).all()


@gpu
@pytest.mark.parametrize("N,C,V,K", [(3, 256, 30000, 20), (100, 256, 50257, 64), (128, 128, 90000, 200), (300, 128, 20000, 50)])
def test_teachers_in_turn_on_one_scratch(N, C, V, K):
    """Calls right behind one another, each with entries, spans and scores in the places of the last one's: every value of every call."""
    cases = [Case(N, C, V, K=K, tau=2.0, seed=s) for s in (1, 2)]
    for c in cases:
        c.x, c.w = cases[0].x, cases[0].w
    plain = [c.forward() for c in cases]
    want = cases[1].want()
    assert float((plain[1][0] - want[0]).abs().max()) < TOL * 4 * max(1.0, float(want[1].abs().max()))
    need = b.bt_op_head_fwd_scratch_bytes(N, C, V, K)
    work = torch.empty(need, dtype=torch.uint8, device=DEV)
    outs = [[torch.full((n,), math.nan, device=DEV) for n in (N, N, 1)] for _ in range(12)]
    aims = [c.aim() for c in cases]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        b.bt_op_head_distill_fwd(cases[0].x, None, cases[0].w, None, aims[i % 2], None, N, C, V, cases[0].inv, *out, work, need)
    b.bt_op_head_check(work)
    for i, out in enumerate(outs):
        assert all(torch.equal(p, q) for p, q in zip(out, plain[i % 2]))
