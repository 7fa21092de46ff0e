"""Pins of the FP8 block and scored-routing oracle: closed forms and other definitions."""

import numpy as np
import pytest
import torch

from oracle import fp8_block as OB, route as ORt


def test_codes_against_torch_casts():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 400)).astype(np.float32) * np.float32(3.0)
    codes, dec = OB.quantize_act(x)
    assert dec.shape == (4, 5)
    for b in range(4):
        p = x[:, 128 * b:128 * (b + 1)]
        enc = np.float32(448.0) / np.abs(p).max(1)
        t = torch.from_numpy(p * enc[:, None]).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        assert np.array_equal(codes[:, 128 * b:128 * (b + 1)], t)
        assert np.array_equal(dec[b], np.float32(1.0) / enc)


def test_small_and_zero_blocks():
    x = np.zeros((3, 256), np.float32)
    x[1, :128] = np.float32(2.0 ** -101)
    x[2, 3] = np.float32(2.0 ** -100)
    codes, dec = OB.quantize_act(x)
    assert not codes[:2].any() and (dec[:, :2] == 1.0).all()
    assert codes[2, 3] == 0x7E and dec[0, 2] < 1e-30 and dec[1, 2] == 1.0


def test_error_of_a_block_is_half_a_step():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((7, 256)).astype(np.float32)
    v = OB.act_values(*OB.quantize_act(x))
    m = np.repeat(np.abs(x).reshape(7, 2, 128).max(2), 128, 1)
    # e4m3: half a step is 2^-4 of the value, 2^-10 of the scale below 2^-6
    assert (np.abs(v - x) <= np.abs(x) * 2.0 ** -4 * 1.0001 + m / 448 * 2.0 ** -10 * 1.0001).all()


def test_weight_blocks_are_the_transposed_matrix_blocks():
    rng = np.random.default_rng(3)
    w = rng.standard_normal((2, 144, 272)).astype(np.float32)
    c, d = OB.quantize_weight(w)
    ct, dt = OB.quantize_weight(w.transpose(0, 2, 1))
    assert np.array_equal(c.transpose(0, 2, 1), ct) and np.array_equal(d.transpose(0, 2, 1), dt)


def test_plain_softmax_routing_is_the_other_oracle_s():
    rng = np.random.default_rng(4)
    lg = rng.standard_normal((33, 16)).astype(np.float32)
    r = OB.route(lg, 4)
    ids = ORt.topk_fast(lg, 4)
    p = ORt.permute(ids, 16)
    assert np.array_equal(r["ids"], ids)
    assert np.array_equal(r["offsets"], p["offsets"])
    assert np.array_equal(r["row_token"], p["row_token"])


def test_routing_worked_example():
    # sigmoid(0) = 1/2 everywhere: the bias alone chooses; the weights are even
    r = OB.route(np.zeros((1, 8), np.float32), 2, scoring="sigmoid",
                 bias=np.array([0, 3, 0, 0, 1, 0, 2, 2]), groups=4, top_groups=2, group_sum=1,
                 scale=2.0)
    assert r["ids"].tolist() == [[1, 6]] and r["w"].tolist() == [[1.0, 1.0]]
    # by two of a group: 3, 0, 1, 4: the last group and the first
    r = OB.route(np.zeros((1, 8), np.float32), 3, scoring="sigmoid", renorm=False,
                 bias=np.array([0, 3, 0, 0, 1, 0, 2, 2]), groups=4, top_groups=2, group_sum=2)
    assert r["ids"].tolist() == [[1, 6, 7]] and r["w"].tolist() == [[0.5, 0.5, 0.5]]


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_against_differences(scoring, renorm):
    rng = np.random.default_rng(5)
    lg = rng.standard_normal((3, 8))
    ids = OB.route(lg, 3, scoring=scoring, renorm=renorm)["ids"]
    g = rng.standard_normal((3, 3))
    d = OB.route_backward(lg, ids, g, scoring, renorm, 1.5)
    # central differences: an error of h^2 / 6 times a third derivative (below 10), and
    # 1e-16 / h of rounding
    h = 1e-5
    for e in range(8):
        up, dn = lg.copy(), lg.copy()
        up[:, e] += h
        dn[:, e] -= h
        f = lambda x: (OB.chosen_weights(x, ids, scoring, renorm, 1.5) * g).sum(1)
        assert np.abs((f(up) - f(dn)) / (2 * h) - d[:, e]).max() < 1e-9


def test_dead_tokens_take_no_rows():
    rng = np.random.default_rng(6)
    lg = rng.standard_normal((5, 4))
    r = OB.route(lg, 2, live=[1, 0, 1, 0, 0])
    assert r["offsets"][-1] == 4 and (r["ids"][[1, 3, 4]] == -1).all()
    assert (r["row_token"][4:] == -1).all() and set(r["row_token"][:4]) == {0, 2}


def test_logits_that_are_no_numbers():
    nan, inf = float("nan"), float("inf")
    lg = np.array([[1, nan, 3, 2], [1, inf, 3, 2], [nan, nan, nan, 0], [nan, -inf, -inf, -inf],
                   [inf, 0, inf, -inf]], np.float32)
    # the choice passes over them, the softmax weights are NaN
    r = OB.route(lg, 2, bias=np.zeros(4))
    assert r["ids"].tolist() == [[2, 3], [1, 0], [3, 0], [1, 2], [0, 2]]
    assert np.isnan(r["w"]).all()
    assert OB.route(lg, 2)["ids"].tolist() == [[2, 3], [1, 2], [3, 0], [1, 2], [0, 2]]
    # sigmoid: a NaN that is not chosen does no harm
    r = OB.route(lg, 2, scoring="sigmoid")
    assert np.isnan(r["w"]).any(1).tolist() == [False, False, True, False, False]
    assert np.isnan(r["w"][2]).all()
    # a group ranks by its numbers as far as they reach
    lg = np.array([[5, nan, 0, 0], [nan, 4, 1, 1]], np.float32)
    for gs, want in ((1, [[0], [1]]), (2, [[2], [2]])):
        r = OB.route(lg, 1, scoring="sigmoid", groups=2, group_sum=gs)
        assert r["ids"].tolist() == want
