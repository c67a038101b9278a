"""The attention sublayer's operators where their arithmetic could give way: scores and biases far beyond a softmax's usual
range, saturated caps, rows that overflow, very wide heads, span tables of another shape, empty arrays; and the device error word."""
import math

import numpy as np
import pytest
import torch

from paper_2606_24780_b200 import binding as b

from gpu_util import DEV
from test_attention_sublayer import A, TOL, Case, attention64, close, lib, planes_of, rand, random_layout, refused, see_matrix, spans_of, ways  # noqa: F401

gpu = pytest.mark.gpu


def given(qkv, d_o, B, T, H, d, cap=0.0, slopes=None, doc=None):
    """A Case of these inputs; qkv [B * T, 3 H d]."""
    case = Case.__new__(Case)
    case.B, case.T, case.H, case.d, case.C = B, T, H, d, H * d
    case.qkv, case.d_o, case.slopes = qkv.contiguous(), d_o.contiguous(), slopes
    see = torch.tensor(see_matrix(doc, None, 0, B, T), device=DEV)
    case.spans = None if doc is None else spans_of(doc, None, 0, B, T)
    case.mod = b.make_attn_mod(cap, slopes, case.spans)
    case.o, case.lse, case.grad, case.size = attention64(case.qkv.double().view(B, T, 3, H, d), see, cap,
                                                         None if slopes is None else slopes.double(), case.d_o.double().view(B, T, H, d))
    size = b.bt_op_attention_mod_scratch_bytes(B, T, case.C, H)
    case.scratch = torch.full((size,), 255, dtype=torch.uint8, device=DEV)
    return case


# ------------------------------------------------------------------------------- CPU: refusals

def test_rows_of_more_than_two_to_the_31_columns_are_refused(lib):
    """128-wide heads, on tcgen05: the columns of a row are counted in 32 bits there."""
    H = (1 << 31) // (3 * 128) + 1
    for heads in (H, 1 << 23):
        refused(2, b.bt_op_attention_mod_fwd, A, None, 1, 1, 128 * heads, heads, b.make_attn_mod(), 2 * A, None, 3 * A, 4 * A, 1 << 62)
        refused(2, b.bt_op_attention_mod_bwd, A, None, 2 * A, 3 * A, 4 * A, None, 1, 1, 128 * heads, heads, b.make_attn_mod(), 5 * A, None,
                6 * A, 1 << 62)


def test_empty_arrays_without_an_address(lib):
    """An empty tensor's address is NULL: with nothing to do, that is no error."""
    none = torch.empty(0)
    assert none.data_ptr() == 0
    cfg = b.make_rope(64)
    for call in (b.bt_op_rope_fwd, b.bt_op_rope_bwd):
        call(None, None, 0, 4, 768, 12, cfg, None, stream=0)
        refused(1, call, A + 4, None, 0, 4, 768, 12, cfg, None)
        refused(1, call, None, None, 0, 4, 768, 7, cfg, None)
    b.bt_op_dropout_fwd(None, None, 0, 0.1, 1, 2, None, stream=0)
    b.bt_op_dropout_bwd(None, 0, 0.1, 1, 2, None, stream=0)
    refused(1, b.bt_op_dropout_bwd, None, 0, 1.0, 1, 2, None)


# ------------------------------------------------------------------------------- scores beyond the usual range

@gpu
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("T", [60, 270])
@pytest.mark.parametrize("value", [150.06, 199.94])
def test_equal_scores_of_a_hundred_thousand(d, T, value):
    """All of q and k the same: every score is the same number, formed by the same operations, whatever its rounding, so every
    key that is read weighs the same.  The values lie between two TF32 numbers, all on the same side: what the rounded
    halves alone give is off by hundreds in the exponent."""
    H = 2
    qkv = rand(1, T, 3 * H * d)
    qkv[:, :2 * H * d] = value
    for cap in (0.0, 1e20):
        case = given(qkv, rand(2, T, H * d), 1, T, H, d, cap)
        for planes, flags in ways(d):
            o, lse = case.forward(planes, flags)
            assert close(o.view_as(case.o), case.o, TOL)
            assert ((lse.double() - case.lse).abs() <= TOL * case.lse.abs()).all()
            assert torch.isfinite(case.backward(planes, flags)).all()


@gpu
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("scale", [100.0, 300.0, 1e6, 1e12])
def test_random_scores_of_a_hundred_thousand_and_more(d, scale):
    """One key takes the row: where its score leads by more than the scores' own errors, the row is that key's value.  An error
    is below 48 * 2^-23 of sum_c |q_c k_c| / sqrt(d) (48 tensor-core additions for 128 columns); a lead of 17 more leaves the others
    less than 1e-7 of the weight."""
    H = 2
    for T in (60, 270):
        qkv = rand(3, T, 3 * H * d)
        qkv[:, :2 * H * d] *= scale
        x = qkv.double().view(T, 3, H, d).permute(1, 2, 0, 3)
        q, k, v = x[0], x[1], x[2]
        below = torch.tril(torch.ones(T, T, dtype=torch.bool, device=DEV))
        s = (q @ k.transpose(1, 2) / math.sqrt(d)).masked_fill(~below, -math.inf)
        off = 48 * 2.0 ** -23 * (q.abs() @ k.abs().transpose(1, 2) / math.sqrt(d)).amax(2)
        two, at = s.topk(2, 2)
        clear = two[..., 0] - two[..., 1] > 2 * off + 17
        assert clear.double().mean() > 0.5
        want = torch.gather(v, 1, at[..., :1].expand(-1, -1, d))
        case = given(qkv, rand(4, T, H * d), 1, T, H, d)
        for planes, flags in ways(d):
            o, lse = case.forward(planes, flags)
            o = o.view(T, H, d).permute(1, 0, 2).double()
            assert torch.isfinite(o).all() and torch.isfinite(lse).all()
            assert close(o[clear], want[clear], TOL)
            assert ((lse[0].double() - two[..., 0]).abs() <= off + 1)[clear].all()


@gpu
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("slope", [1e4, -1e4, 1e7, -1e7, 1e12, -1e30])
def test_biases_beyond_every_score(d, slope):
    """A slope that outweighs all scores leaves each query its own key, a negative one the first key of the sequence.  The bias of
    neighbouring keys differs by more than one rounding of the largest, so the weights are 0 and 1 in FP32 as well."""
    H = 2
    slopes = torch.full((H,), slope, device=DEV)
    for T in (60, 270):
        for cap in (0.0, 30.0):
            case = given(rand(5, T, 3 * H * d), rand(6, T, H * d), 1, T, H, d, cap, slopes)
            for planes, flags in ways(d):
                o, lse = case.forward(planes, flags)
                assert close(o.view_as(case.o), case.o, TOL)
                assert torch.isfinite(lse).all()


@gpu
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("slope", [100.0, 1e4, 1e7, 1e12])
def test_a_steep_bias_leaves_the_own_key_its_score(d, slope):
    """The distance to the own key is zero, and so is its bias, whatever the slope; the row's lse is that one score, and the
    gradients are those of a query that reads a single key."""
    H = 2
    slopes = torch.full((H,), slope, device=DEV)
    for T in (60, 270):
        for cap in (0.0, 30.0):
            case = given(rand(5, T, 3 * H * d), rand(6, T, H * d), 1, T, H, d, cap, slopes)
            for planes, flags in ways(d):
                case.check(planes, flags)


@gpu
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("signs", [(1, 1), (1, -1), (0, 0)])
def test_rows_out_of_fp32s_range_are_not_taken_for_rows_that_read_nothing(d, signs):
    """q and k of 5e19: every product is beyond FP32 (to +inf, to -inf, or of either sign), so no score is a number.  The rows
    that read them have no value; rows of padding, which read nothing, are zero with lse -inf as always."""
    H = 2
    for T in (60, 270):
        qkv = rand(7, T, 3, H * d)
        for part, sign in enumerate(signs):
            size = 5e19 * (0.5 + torch.rand(T, H * d, generator=torch.Generator(DEV).manual_seed(8 + part), device=DEV))
            qkv[:, part] = size * (sign or torch.sign(qkv[:, part]))
        doc = np.zeros((1, T), np.int32)
        doc[0, T // 2:] = -1
        case = given(qkv.view(T, -1), rand(9, T, H * d), 1, T, H, d, doc=doc)
        for planes, flags in ways(d):
            o, lse = case.forward(planes, flags)
            assert torch.isnan(lse[:, :, :T // 2]).all() and torch.isnan(o[:T // 2]).all()
            assert (lse[:, :, T // 2:] == -math.inf).all()


# ------------------------------------------------------------------------------- saturated caps

@gpu
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("size", [0.6, 2.0, 4.5, 6.5, 10.0, 20.0])
def test_gradients_of_scores_several_caps_out(d, size):
    """All |u| = |score| / cap within a fifth of `size`.  du: a score's 48 additions of up to 2^-23 of it each, its operands' splits
    and scaling 2^-21, an exponential's argument 2 |u| log2 e rounded by 2^-24 of itself: 53 * 2^-23 |u|.  1 - tanh^2(u) moves by
    2 du of itself, a weight by cap (1 - tanh^2) du and by the roundings of z and lse, three of 2^-24 of cap + log T.  The rest of a
    gradient is 1e-5 as everywhere."""
    H = 2
    for T in (60, 270):
        for cap in (1.0, 25.0):
            du = 53 * 2.0 ** -23 * 1.2 * size
            tol = 2 * du + cap / math.cosh(0.8 * size) ** 2 * du + 3 * 2.0 ** -24 * (cap + math.log(T)) + TOL
            c = math.sqrt(size * cap / math.sqrt(d))
            qkv = rand(11, T, 3, H, d)
            swing = 0.975 + 0.05 * torch.rand(2, T, H, 1, generator=torch.Generator(DEV).manual_seed(12), device=DEV)
            sign = torch.sign(qkv[:, 0, :, :1])
            qkv[:, 0] = c * (1 + 0.05 * qkv[:, 0].clamp(-1, 1)) * swing[0] * sign
            qkv[:, 1] = c * (1 + 0.05 * qkv[:, 1].clamp(-1, 1)) * swing[1]
            u = torch.einsum("ihc,jhc->hij", qkv[:, 0].double(), qkv[:, 1].double()) / math.sqrt(d) / cap
            assert 0.8 * size < float(u.abs().min()) and float(u.abs().max()) < 1.2 * size
            case = given(qkv.view(T, -1), rand(13, T, H * d), 1, T, H, d, cap)
            # 1 - tanh^2 in 64 bits keeps 1e-16 / 4e^-2|u| of itself: enough up to |u| = 12; beyond, the gradients of q and k scale as
            # 4 e^-2|u|, which is taken out of the comparison's weights below
            if size > 10:
                t = 1 / torch.cosh(u) ** 2
                case.grad = gradients_with(case, u, t, cap)
            for planes, flags in ways(d):
                dqkv = case.backward(planes, flags).view_as(case.grad)
                for n in range(3):
                    got, want = dqkv[0, :, n].double(), case.grad[0, :, n]
                    assert float((got - want).norm()) <= tol * max(float(want.norm()), case.size[n]), "qkv"[n]


def gradients_with(case, u, t, cap):
    """attention64's gradients for one causal sequence, with 1 - tanh^2 given."""
    T, H, d = case.T, case.H, case.d
    q, k, v = case.qkv.double().view(T, 3, H, d).permute(1, 2, 0, 3)
    g = case.d_o.double().view(T, H, d).permute(1, 0, 2)
    z = (cap * torch.tanh(u)).masked_fill(~torch.tril(torch.ones(T, T, dtype=torch.bool, device=DEV)), -math.inf)
    p = torch.softmax(z, 2)
    o = p @ v
    ds = p * (g @ v.transpose(1, 2) - (g * o).sum(2, keepdim=True)) * t / math.sqrt(d)
    w = p ** 2 * ((g @ v.transpose(1, 2)) ** 2 + (g * o).sum(2, keepdim=True) ** 2) * t ** 2 / d
    case.size = [float((w @ k ** 2).sum().sqrt()), float((w.transpose(1, 2) @ q ** 2).sum().sqrt()), 0.0]
    return torch.stack((ds @ k, ds.transpose(1, 2) @ q, p.transpose(1, 2) @ g)).permute(2, 0, 1, 3)[None]


# ------------------------------------------------------------------------------- rotary positions of wide heads

@gpu
@pytest.mark.parametrize("H,d,rot,inter", [
    (1, 65532, 4, False), (1, 65536, 2, True), (32, 16380, 2, False), (8192, 1000, 6, False), (1, 1 << 20, 8, True), (3, 1 << 20, 8, False),
    (1 << 15, 128, 128, False), (1, 1 << 26, 8, False)])
def test_rope_of_heads_hardly_turned(H, d, rot, inter):
    """Every column is written once, from its own place, however many there are: none of y's old contents stay, and what does not turn
    is copied bit for bit."""
    C, N = H * d, 2 if H * d < 1 << 24 else 1
    x = rand(1, N, 3 * C)
    pos = torch.tensor([5, 1 << 20][:N], dtype=torch.int32, device=DEV)
    y = torch.full_like(x, math.nan)
    b.bt_op_rope_fwd(x, pos, N, 1, C, H, b.make_rope(rot, inter), y)
    got, was = y.view(N, 3, H, d), x.view(N, 3, H, d)
    assert torch.equal(got[:, 2], was[:, 2]) and torch.equal(got[:, :2, :, rot:], was[:, :2, :, rot:])
    for i in range(rot // 2):
        u, w = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        a = pos.double() * 10000.0 ** (-2.0 * i / rot)
        c, s = torch.cos(a)[:, None, None], torch.sin(a)[:, None, None]
        p, q = was[:, :2, :, u].double(), was[:, :2, :, w].double()
        off = 8 * 2.0 ** -24 * (p.abs() + q.abs())      # two products and a sum, sine and cosine within 2^-22
        assert ((got[:, :2, :, u] - (p * c - q * s)).abs() <= off).all() and ((got[:, :2, :, w] - (p * s + q * c)).abs() <= off).all()


# ------------------------------------------------------------------------------- span tables of another shape

@gpu
@pytest.mark.parametrize("d", [16, 32, 64, 128])
def test_spans_of_another_shape_reach_no_other_sequence(d):
    """A table of 2 x 512 positions has the size of one of 4 x 256 or 8 x 128, and its ranges go past their ends.  What a row reads
    that way is not specified, but it lies inside its sequence: the last sequence's outputs do not change with the others'
    contents, and the call ends.  Tables of arbitrary numbers likewise."""
    H = 2
    wrong = spans_of(None, None, 0, 2, 512)
    noise = torch.randint(-2 ** 31, 2 ** 31 - 1, (wrong.numel() // 4,), generator=torch.Generator(DEV).manual_seed(14), dtype=torch.int32, device=DEV)
    small = torch.randint(-600, 600, noise.shape, generator=torch.Generator(DEV).manual_seed(15), dtype=torch.int32, device=DEV)
    for B, T in ((4, 256), (8, 128), (3, 100), (2, 333)):
        for table in (wrong, noise.view(torch.uint8), small.view(torch.uint8)):
            case = given(rand(16, B * T, 3 * H * d), rand(17, B * T, H * d), B, T, H, d)
            case.mod = b.make_attn_mod(20.0, None, table)
            for planes, flags in ways(d):
                got = [t.clone() for t in (*case.forward(planes, flags), case.backward(planes, flags))]
                was = case.qkv.clone()
                case.qkv[:(B - 1) * T] = rand(18, (B - 1) * T, 3 * H * d)
                again = (*case.forward(planes, flags), case.backward(planes, flags))
                case.qkv = was
                for x, y in zip(got, again):
                    x, y = x.reshape(B, -1)[-1], y.reshape(B, -1)[-1]
                    assert torch.equal(torch.nan_to_num(x, 0.0, 1.0, -1.0), torch.nan_to_num(y, 0.0, 1.0, -1.0))


# ------------------------------------------------------------------------------- the error word, gradients as differences

@gpu
@pytest.mark.parametrize("d,T", [(16, 60), (16, 300), (32, 200), (64, 200), (128, 140)])
def test_the_error_word_is_reported_and_cleared(d, T):
    """A word left in the scratch as a wait that ran out leaves it is an error with that code; every kernel family's forward and
    backward begin with a clear one."""
    case = Case(2, T, 2, d, mean=50, cap=30.0)
    B, C, H = case.B, case.C, case.H
    o, lse, dqkv = torch.empty(B * T, C, device=DEV), torch.empty(B, H, T, device=DEV), torch.empty(B * T, 3 * C, device=DEV)
    o_in, lse_in = case.o.reshape(B * T, C).float().contiguous(), case.lse.float().contiguous()
    word = case.scratch[:4].view(torch.int32)
    for planes, flags in ways(d):
        forms = [(None, planes_of(t)) if planes else (t, None) for t in (case.qkv, case.d_o)]
        for call in (lambda: b.bt_op_attention_mod_fwd(*forms[0], B, T, C, H, case.mod, o, None, lse, case.scratch, case.scratch.numel(), flags),
                     lambda: b.bt_op_attention_mod_bwd(*forms[0], o_in, lse_in, *forms[1], B, T, C, H, case.mod, dqkv, None, case.scratch,
                                                       case.scratch.numel(), flags)):
            word.fill_(4711)
            with pytest.raises(b.BtError, match="4711") as e:
                b.bt_op_attention_mod_check(case.scratch)
            assert b.STATUS[e.value.status] == "BT_ERR_DEVICE_TIMEOUT"
            call()
            b.bt_op_attention_mod_check(case.scratch)
            assert int(word) == 0


@gpu
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("mod", [dict(), dict(mean=60, prefix=10, cap=5.0, slope=True), dict(cap=1.0, scale=1.5), dict(window=20, slope=True)])
def test_gradients_against_differences_of_the_definition(d, mod):
    """The gradient along u, against (f(x + h u) - f(x - h u)) / 2h of f = sum(o * g) in 64 bits: no gradient formula on that side.
    With h = 2^-12 and scores of a few units the cubic term is below 1e-6 of the derivative's scale, and 64-bit rounding
    below 1e-16 * |f| / h.  A gradient off by 1e-5 of its norm moves the derivative along a normal u by that times a
    normal number: six of them at most."""
    mod = dict(mod)
    case = Case(1, 150, 2, d, **mod)
    B, T, H = case.B, case.T, case.H
    slopes = None if case.slopes is None else case.slopes.double()
    if "mean" in mod:
        doc, mark = random_layout(np.random.default_rng(7 * T), B, T, mod["mean"], 0, mod["prefix"])       # the Case's own
        see = see_matrix(doc, mark, 0, B, T)
    else:
        see = see_matrix(None, None, mod.get("window", 0), B, T)
    see = torch.tensor(see, device=DEV)
    x, g, h = case.qkv.double().view(B, T, 3, H, d), case.d_o.double().view(B, T, H, d), 2.0 ** -12
    for seed in range(3):
        u = torch.randn(x.shape, generator=torch.Generator(DEV).manual_seed(20 + seed), device=DEV, dtype=torch.float64)
        f = [float((attention64(x + sign * h * u, see, mod.get("cap", 0.0), slopes)[0] * g).sum()) for sign in (1.0, -1.0)]
        for planes, flags in ways(d):
            grad = case.backward(planes, flags).double().view(x.shape)
            assert abs(float((grad * u).sum()) - (f[0] - f[1]) / (2 * h)) <= 6 * TOL * float(grad.norm())
