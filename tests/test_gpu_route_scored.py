"""Scored routing and its gradient on the GPU against the float64 oracle.

Choices and permutations must be equal (both sides compare float64 scores; equal
logits give equal scores on each side).  A weight is float64 rounded once to float32:
2^-24 of it.  A gradient in float32 likewise, in bf16 2^-8; the float64 arithmetic
before that rounding is off by less than 2^-40 of its terms."""

import numpy as np
import pytest
import torch

from oracle import fp8_block as OB
from paper_2607_15810_amd import ops
from paper_2607_15810_amd import quads as Q

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.lib()
    yield


def np_of(t):
    return t.detach().cpu().numpy()


def check(got, ref):
    ids, w, offs, tok, inv = [np_of(t) for t in got]
    assert np.array_equal(ids, ref["ids"])
    assert np.array_equal(offs, ref["offsets"])
    assert np.array_equal(tok, ref["row_token"])
    assert np.array_equal(inv, ref["inv_row"])
    d = np.abs(w.astype(np.float64) - ref["w"])
    assert (d <= ref["w"] * 2.0 ** -23.99 + 2.0 ** -149).all(), d.max()


CASES = [
    # T, E, k, router
    (1, 1, 1, dict()),
    (1, 8, 8, dict(scoring="sigmoid")),
    (1, 256, 8, dict(scoring="sigmoid", bias=True, groups=8, top_groups=4, group_sum=2, scale=2.5)),
    (3, 60, 4, dict(renorm=False)),
    (64, 128, 8, dict(bias=True)),
    (65, 128, 6, dict(scoring="sigmoid", groups=4, top_groups=2, group_sum=1)),
    (255, 160, 6, dict(bias=True, groups=8, top_groups=3, group_sum=2, scale=16.0, renorm=False)),
    (256, 96, 8, dict(scoring="sigmoid", bias=True)),
    (257, 256, 32, dict(scoring="sigmoid", bias=True, groups=64, top_groups=20, group_sum=2)),
    (700, 64, 8, dict()),
    (1025, 129, 3, dict(scoring="sigmoid", renorm=False)),
    (300, 384, 8, dict(scoring="sigmoid", bias=True, groups=1)),
    (70, 1024, 10, dict(bias=True, groups=16, top_groups=2, group_sum=2)),
    (520, 513, 1, dict()),
    (40, 24, 2, dict(scoring="sigmoid", bias=True, groups=24, top_groups=2, group_sum=1)),
]


@pytest.mark.parametrize("live", [None, "some", "none"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", CASES, ids=[f"t{c[0]}_e{c[1]}_k{c[2]}" for c in CASES])
def test_route(case, dtype, live):
    T, E, k, kw = case
    kw = dict(kw)
    rng = np.random.default_rng(T * 1000 + E)
    # rows E + 3 apart; bf16 gives many equal logits
    wide = torch.from_numpy(rng.standard_normal((T, E + 3)).astype(np.float32)).to(DEV).to(dtype)
    lg = wide[:, :E]
    if kw.pop("bias", False):
        b = torch.from_numpy((0.1 * rng.standard_normal(E)).astype(np.float32))
        kw["bias"] = b
    lv = None
    if live:
        lv = (rng.random(T) < 0.6) if live == "some" else np.zeros(T, bool)
    okw = dict(kw, bias=np_of(kw["bias"]) if "bias" in kw else None)
    ref = OB.route(np_of(lg.float()), k, live=lv, **okw)
    if "bias" in kw:
        kw["bias"] = kw["bias"].to(DEV)
    got = ops.route_scored(lg, k, live=None if lv is None else torch.from_numpy(lv).to(DEV), **kw)
    check(got, ref)
    # the gradient
    gw = torch.from_numpy(rng.standard_normal((T, k)).astype(np.float32)).to(DEV)
    sc, rn, sl = kw.get("scoring", "softmax"), kw.get("renorm", True), kw.get("scale", 1.0)
    gr = ops.route_scored_backward(lg, got[0], gw, scoring=sc, renorm=rn, scale=sl)
    assert gr.dtype == dtype
    if T * E * E <= 2 ** 24:
        d = OB.route_backward(np_of(lg.float()), ref["ids"], np_of(gw), sc, rn, sl)
        half = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8 * (1 + 2.0 ** -15)
        err = np.abs(np_of(gr.float()).astype(np.float64) - d)
        assert (err <= half * np.abs(d) * 1.001 + abs(sl) * 2.0 ** -38).all()


def test_ties_and_extremes():
    E = 64
    lg = torch.zeros((6, E), device=DEV)
    lg[1, :] = -float("inf")                       # every expert masked
    lg[2, 5:] = -float("inf")                      # fewer than k left
    lg[3, 10] = lg[3, 40] = 90.0                   # saturated: sigmoid 1 twice
    lg[4, :] = torch.finfo(torch.float32).min
    lg[5, 33] = 1.0
    for kw in (dict(), dict(scoring="sigmoid"), dict(renorm=False),
               dict(scoring="sigmoid", groups=8, top_groups=2, group_sum=2)):
        with np.errstate(over="ignore"):
            ref = OB.route(np_of(lg), 8, **kw)
        check(ops.route_scored(lg, 8, **kw), ref)


@pytest.mark.parametrize("E,groups", [(64, 1), (96, 4), (128, 8), (160, 5), (256, 8), (512, 16), (1024, 1)])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_scores_that_float32_cannot_tell_apart(E, groups, scoring):
    """Neighbouring float32 logits at magnitudes where the float32 scores (and the
    sums of two) of different experts coincide, and biases that move them back."""
    rng = np.random.default_rng(E + groups)
    T = 130
    base = rng.choice([-9.0, 0.25, 3.0, 6.0], (T, 1)).astype(np.float32)
    step = rng.integers(0, 9, (T, E)).astype(np.float32) * np.float32(2.0 ** -21)
    lg = base + step * np.abs(base)
    for bias in (np.zeros(E, np.float32), rng.choice([0, 2.0 ** -30, -2.0 ** -30], E).astype(np.float32)):
        kw = dict(scoring=scoring, groups=groups, top_groups=max(1, groups // 2), group_sum=2)
        ref = OB.route(lg, 8, bias=bias, **kw)
        check(ops.route_scored(torch.from_numpy(lg).to(DEV), 8, bias=torch.from_numpy(bias).to(DEV),
                               **kw), ref)


def test_nan_stays_in_its_row():
    rng = np.random.default_rng(3)
    lg = torch.from_numpy(rng.standard_normal((9, 128)).astype(np.float32)).to(DEV)
    clean = ops.route_scored(lg, 4, scoring="sigmoid", groups=4, top_groups=2)
    bad = lg.clone()
    bad[4, 7:] = float("nan")
    for sc in ("sigmoid", "softmax"):
        ids, w, offs, tok, inv = ops.route_scored(bad, 4, scoring=sc, groups=4, top_groups=2)
        i = np_of(ids)
        assert ((i >= 0) & (i < 128)).all() and all(len(set(r)) == 4 for r in i.tolist())
        assert int(offs[-1]) == 36
    ids = ops.route_scored(bad, 4, scoring="sigmoid", groups=4, top_groups=2)[0]
    keep = [t for t in range(9) if t != 4]
    assert torch.equal(ids[keep], clean[0][keep])
    assert set(np_of(ids[4]).tolist()) <= set(range(0, 7)) | set(range(0, 128))


def test_no_tokens():
    ids, w, offs, tok, inv = ops.route_scored(torch.zeros((0, 8), device=DEV), 2)
    assert ids.shape == (0, 2) and not offs.any()
    g = ops.route_scored_backward(torch.zeros((0, 8), device=DEV), ids, w)
    assert g.shape == (0, 8)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient_of_one_renormalised_expert_is_zero(scoring, dtype):
    """Its weight is the scale whatever the logits: no rounding is left in the gradient."""
    lg = torch.randn((300, 96), device=DEV).to(dtype)
    ids, w, *_ = ops.route_scored(lg, 1, scoring=scoring, scale=2.5)
    assert (w == 2.5).all()
    grad = ops.route_scored_backward(lg, ids, torch.randn((300, 1), device=DEV), scoring=scoring,
                                     scale=2.5)
    assert not grad.any()


def test_gradient_leaves_the_gaps_between_rows():
    T, E, k, ld = 5, 24, 3, 40
    lg = torch.randn((T, E), device=DEV)
    ids = ops.route_scored(lg, k)[0]
    gw = torch.randn((T, k), device=DEV)
    out = torch.full((T, ld), 7.0, device=DEV)
    Q.call("moe_route_scored_backward", lg.data_ptr(), Q.QD_DTYPE_F32, E, T, E, k, 0, 1, 1.0,
           ids.data_ptr(), gw.data_ptr(), out.data_ptr(), ld,
           torch.cuda.current_stream().cuda_stream)
    assert (out[:, E:] == 7.0).all()
    assert torch.equal(out[:, :E], ops.route_scored_backward(lg, ids, gw))


def test_two_streams_and_a_graph():
    T, E, k = 300, 128, 8
    kw = dict(scoring="sigmoid", groups=8, top_groups=4, group_sum=2)
    a, b = torch.randn((T, E), device=DEV), torch.randn((T, E), device=DEV)
    want = [ops.route_scored(x, k, **kw) for x in (a, b)]
    torch.cuda.synchronize()
    got = []
    for x in (a, b):
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            got.append(ops.route_scored(x, k, **kw))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(g, w))
    x = a.clone()
    ops.route_scored(x, k, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.route_scored(x, k, **kw)
    for src, w in ((b, want[1]), (a, want[0]), (b, want[1])):
        x.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, w))
        assert torch.equal(ops.route_scored(src, k, **kw)[0], w[0])


BROKEN = [
    # T, E, k, router (bias: -3 on the last expert, so that +inf there is not chosen)
    (13, 8, 3, dict()), (13, 8, 3, dict(bias=True)),
    (64, 128, 8, dict(groups=8, top_groups=4, group_sum=2)),
    (65, 128, 6, dict(bias=True, groups=4, top_groups=2, group_sum=1)),
    (300, 256, 8, dict(bias=True, groups=8, top_groups=4, group_sum=2)),
    (70, 60, 4, dict(bias=True, groups=20, top_groups=9, group_sum=2)),
    (40, 96, 8, dict(groups=6, top_groups=2, group_sum=2)),
    (26, 1024, 10, dict(bias=True)), (13, 513, 4, dict()),
]


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", BROKEN, ids=[f"t{c[0]}_e{c[1]}_k{c[2]}" for c in BROKEN])
def test_logits_that_are_no_numbers(case, dtype, scoring, renorm):
    """A NaN is chosen after every number; a softmax row with a NaN or +inf anywhere has NaN
    weights, and a choice of its numbers; no other row changes."""
    T, E, k, kw = case
    kw = dict(kw, scoring=scoring, renorm=renorm)
    rng = np.random.default_rng(E + T)
    x = rng.standard_normal((T, E)).astype(np.float32)
    nan, inf = np.float32("nan"), np.float32("inf")
    low = x.argmin(1)
    for t in range(T):
        at = t % 13
        if at == 1:                                # on an expert that would not be chosen
            x[t, low[t]] = nan
        elif at == 2:
            x[t, E - 1] = inf
        elif at == 3:                              # on the one that would be first
            x[t, x[t].argmax()] = nan
        elif at == 4:
            x[t, rng.permutation(E)[2:]] = nan
        elif at == 5:
            x[t] = nan
        elif at == 6:
            x[t, [1, E - 2]] = inf
        elif at == 7:
            x[t, 0], x[t, E // 2] = nan, inf
        elif at == 8:
            x[t] = -inf
            x[t, 1] = nan
        elif at == 9:
            x[t] = -inf
            x[t, 2] = inf
        elif at == 10:                             # the lowest group of experts and some of the next
            x[t, :E // 3] = nan
        elif at == 11:
            x[t] = inf
    lg = torch.from_numpy(x).to(DEV).to(dtype)
    b = None
    if kw.pop("bias", False):
        b = (0.1 * rng.standard_normal(E)).astype(np.float32)
        b[E - 1] = -3.0
    ref = OB.route(np_of(lg.float()), k, bias=b, **kw)
    got = ops.route_scored(lg, k, bias=None if b is None else torch.from_numpy(b).to(DEV), **kw)
    ids, w, offs, tok, inv = [np_of(t) for t in got]
    assert np.array_equal(ids, ref["ids"])
    assert np.array_equal(offs, ref["offsets"])
    assert np.array_equal(tok, ref["row_token"]) and np.array_equal(inv, ref["inv_row"])
    if scoring == "softmax":
        broken = (np.isnan(x) | np.isposinf(x)).any(1)
        assert np.isnan(w[broken]).all() and not np.isnan(w[~broken]).any()
    assert np.array_equal(np.isnan(w), np.isnan(ref["w"]))
    fine = ~np.isnan(w)
    d = np.abs(w.astype(np.float64) - ref["w"])[fine]
    assert (d <= ref["w"][fine] * 2.0 ** -23.99 + 2.0 ** -149).all()
    # NaN after every number of the groups that take part
    if kw.get("groups", 1) == 1:
        numbers = (~np.isnan(x)).sum(1)
        for t in range(T):
            assert np.isnan(x[t, ids[t]]).sum() == max(0, k - numbers[t])


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,E", [(9, 40), (300, 128), (12, 384)])
def test_gradient_of_dead_tokens_over_stale_logits_is_zero(T, E, dtype, scoring, renorm):
    """A batch padded to its graph's size: the logits behind the live tokens are anything."""
    k = 3
    lg = torch.randn((T, E), device=DEV).to(dtype)
    live = torch.ones(T, dtype=torch.uint8, device=DEV)
    live[T // 2:] = 0
    clean = ops.route_scored(lg, k, scoring=scoring, renorm=renorm, live=live)
    gw = torch.randn((T, k), device=DEV)
    want = ops.route_scored_backward(lg, clean[0], gw, scoring=scoring, renorm=renorm)
    bits_of = torch.int32 if dtype == torch.float32 else torch.int16
    assert not want[T // 2:].view(bits_of).any()                  # +0, not -0
    for fill in (float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).min):
        lg[T // 2:] = fill
        lg[T - 1, : E // 2] = 1.0
        gw[T // 2:] = fill
        ids = ops.route_scored(lg, k, scoring=scoring, renorm=renorm, live=live)[0]
        assert torch.equal(ids, clean[0])
        got = ops.route_scored_backward(lg, ids, gw, scoring=scoring, renorm=renorm)
        assert torch.equal(got.view(bits_of), want.view(bits_of))


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,E,k", [(12, 24, 1), (16, 128, 4), (12, 384, 8)])
def test_gradient_where_the_weights_are_nan(T, E, k, dtype, scoring, renorm):
    """NaN at the chosen experts (softmax without renormalisation: at every one) of a token
    whose weights are NaN, zeros at the others, and every other token as it was."""
    rng = np.random.default_rng(E)
    x = torch.from_numpy(rng.standard_normal((T, E)).astype(np.float32)).to(dtype).float().numpy()
    gw = rng.standard_normal((T, k)).astype(np.float32)
    back = lambda ids, lg: np_of(ops.route_scored_backward(
        lg, ids, torch.from_numpy(gw).to(DEV), scoring=scoring, renorm=renorm).float())
    lg = torch.from_numpy(x).to(DEV).to(dtype)
    clean = back(ops.route_scored(lg, k, scoring=scoring, renorm=renorm)[0], lg)
    x[1, x[1].argmin()] = np.nan                   # not chosen
    x[3, :] = np.nan
    x[4, 5] = np.inf
    x[5] = -np.inf
    x[5, 2] = np.nan
    x[6, x[6].argmax()] = np.nan
    lg = torch.from_numpy(x).to(DEV).to(dtype)
    ids = ops.route_scored(lg, k, scoring=scoring, renorm=renorm)[0]
    got = back(ids, lg)
    with np.errstate(invalid="ignore"):
        want = OB.route_backward(x, np_of(ids), gw, scoring, renorm)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    if scoring == "softmax":
        assert np.isnan(got[[1, 3, 4, 5, 6]]).sum(1).tolist() == [k if renorm else E] * 5
    same = [0, 2] + list(range(7, T))
    assert np.array_equal(got[same], clean[same])
    half = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8 * (1 + 2.0 ** -15)
    fine = ~np.isnan(want)
    err = np.abs(got.astype(np.float64) - want)[fine]
    assert (err <= half * np.abs(want[fine]) * 1.001 + 2.0 ** -38).all()


def test_bf16_gradient_is_rounded_once():
    """Sigmoid at 0: the gradient is scale * grad_w / 4, exact in float64.  Products next to the
    middle of two bf16 numbers, nearer than float32 can tell."""
    T, E = 512, 8
    scale = np.float32(1.6369615793)
    m = np.arange(T * E).reshape(T, E)
    middle = (1 + (2 * (m % 128) + 1) * 2.0 ** -8) * 2.0 ** (m // 128 - 16)
    gw = (middle / np.float64(scale)).astype(np.float32) * np.where(m % 3, 1, -1).astype(np.float32)
    v = np.float64(scale) * gw.astype(np.float64) / 4
    step = 2.0 ** (np.floor(np.log2(np.abs(v))) - 7)
    want = np.round(v / step) * step               # to even, one rounding
    by_float = (v.astype(np.float32) / step)
    assert (np.round(by_float) * step != want).sum() > 200
    ids = torch.arange(E, dtype=torch.int32, device=DEV).repeat(T, 1)
    got = ops.route_scored_backward(torch.zeros((T, E), dtype=torch.bfloat16, device=DEV), ids,
                                    torch.from_numpy(gw).to(DEV), scoring="sigmoid", renorm=False,
                                    scale=float(scale))
    assert np.array_equal(np_of(got.float()).astype(np.float64), want)
    # beyond bf16's largest number, and below its smallest
    big = torch.tensor([[3.39e38, -3.3961776e38, 3.4028235e38, 1e-45]], device=DEV)
    got = ops.route_scored_backward(torch.zeros((1, 4), dtype=torch.bfloat16, device=DEV),
                                    ids[:1, :4].contiguous(), big, scoring="sigmoid", renorm=False,
                                    scale=4.0)
    assert torch.equal(got, big.to(torch.bfloat16))


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,E,k", [(20, 200, 8), (9, 256, 32), (14, 257, 8), (11, 384, 6),
                                   (9, 512, 8), (10, 513, 1), (9, 1024, 32)])
def test_gradient_of_many_experts(T, E, k, dtype, scoring, renorm):
    """Every width of the kernel, rows E + 5 apart, against the oracle."""
    rng = np.random.default_rng(T + E)
    wide = torch.from_numpy((2 * rng.standard_normal((T, E + 5))).astype(np.float32)).to(DEV).to(dtype)
    lg = wide[:, :E]
    live = rng.random(T) < 0.8
    ids = ops.route_scored(lg, k, scoring=scoring, renorm=renorm, scale=2.5,
                           live=torch.from_numpy(live).to(DEV))[0]
    gw = rng.standard_normal((T, k)).astype(np.float32)
    got = np_of(ops.route_scored_backward(lg, ids, torch.from_numpy(gw).to(DEV), scoring=scoring,
                                          renorm=renorm, scale=2.5).float()).astype(np.float64)
    want = OB.route_backward(np_of(lg.float()), np_of(ids), gw, scoring, renorm, 2.5)
    half = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
    assert (np.abs(got - want) <= half * np.abs(want) * 1.001 + 2.5 * 2.0 ** -38).all()
    assert not got[~live].any()
