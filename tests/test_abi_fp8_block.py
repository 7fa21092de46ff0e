"""Host-only checks of the scored router and the FP8 block calls: every refusal comes
before a launch, with its documented status."""

import pytest
import torch

from paper_2607_15810_amd import ops
from paper_2607_15810_amd import quads as Q

P = 1 << 20                # an aligned, never-dereferenced address
BIG = 1 << 30


def route(**kw):
    a = dict(logits=P, dtype=1, ld=16, T=4, E=16, k=2, scoring=0, bias=None, groups=1, top=1,
             gsum=1, renorm=1, scale=1.0, live=None, ids=P, w=P, offs=P, tok=P, inv=P, ws=P,
             n=BIG)
    a.update(kw)
    return Q.raw("moe_route_scored_permute", *a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), Q.QD_ERR_DTYPE), (dict(scoring=2), Q.QD_ERR_DTYPE),
    (dict(ld=15), Q.QD_ERR_SHAPE), (dict(T=-1), Q.QD_ERR_SHAPE), (dict(E=0), Q.QD_ERR_SHAPE),
    (dict(E=1025, ld=1025), Q.QD_ERR_SHAPE), (dict(k=0), Q.QD_ERR_SHAPE),
    (dict(k=17), Q.QD_ERR_SHAPE), (dict(E=64, ld=64, k=33), Q.QD_ERR_SHAPE),
    (dict(T=1 << 31), Q.QD_ERR_SHAPE), (dict(groups=3), Q.QD_ERR_SHAPE),
    (dict(groups=0), Q.QD_ERR_SHAPE), (dict(E=128, ld=128, groups=128), Q.QD_ERR_SHAPE),
    (dict(groups=4, top=5), Q.QD_ERR_SHAPE), (dict(groups=4, top=0), Q.QD_ERR_SHAPE),
    (dict(gsum=3), Q.QD_ERR_SHAPE), (dict(groups=16, top=2, gsum=2), Q.QD_ERR_SHAPE),
    (dict(groups=8, top=1, k=3), Q.QD_ERR_SHAPE), (dict(scale=float("inf")), Q.QD_ERR_SHAPE),
    (dict(scale=float("nan")), Q.QD_ERR_SHAPE), (dict(renorm=2), Q.QD_ERR_SHAPE),
    (dict(logits=None), Q.QD_ERR_NULL), (dict(offs=None), Q.QD_ERR_NULL),
    (dict(inv=None), Q.QD_ERR_NULL), (dict(T=257, ws=None), Q.QD_ERR_WORKSPACE),
    (dict(T=257, n=16), Q.QD_ERR_WORKSPACE), (dict(logits=P + 4), Q.QD_ERR_ALIGN),
    (dict(bias=P + 4), Q.QD_ERR_ALIGN), (dict(ws=P + 8), Q.QD_ERR_ALIGN),
])
def test_route_refusals(kw, want):
    assert route(**kw) == want


def test_route_backward_refusals():
    def call(**kw):
        a = dict(logits=P, dtype=0, ld=16, T=4, E=16, k=2, scoring=1, renorm=1, scale=1.0, ids=P,
                 g=P, out=P, ldg=16)
        a.update(kw)
        return Q.raw("moe_route_scored_backward", *a.values(), None)
    assert call(T=0) == Q.QD_OK
    assert call(ldg=8) == Q.QD_ERR_SHAPE
    assert call(k=33, E=64, ld=64, ldg=64) == Q.QD_ERR_SHAPE
    assert call(g=None) == Q.QD_ERR_NULL
    assert call(out=P + 2) == Q.QD_ERR_ALIGN
    assert call(dtype=5) == Q.QD_ERR_DTYPE


def test_quantiser_refusals():
    r = lambda *a: Q.raw("fp8_block_quantize_act", *a, None)
    assert r(P, 0, 4, 24, 24, P, P) == Q.QD_ERR_SHAPE
    assert r(P, 0, 4, 32, 16, P, P) == Q.QD_ERR_SHAPE
    assert r(P, 0, 4, 32, 36, P, P) == Q.QD_ERR_SHAPE
    assert r(P, 3, 4, 32, 32, P, P) == Q.QD_ERR_DTYPE
    assert r(P, 0, -1, 32, 32, P, P) == Q.QD_ERR_SHAPE
    assert r(None, 0, 4, 32, 32, P, P) == Q.QD_ERR_NULL
    assert r(P + 8, 0, 4, 32, 32, P, P) == Q.QD_ERR_ALIGN
    assert r(None, 0, 0, 32, 32, None, None) == Q.QD_OK
    r = lambda *a: Q.raw("fp8_block_quantize_weight", *a, None)
    assert r(P, 0, 2, 16, 24, P, P, None, None) == Q.QD_ERR_SHAPE
    assert r(P, 0, 2, 8, 32, P, P, P, P) == Q.QD_ERR_SHAPE          # transposed: rows % 16
    assert r(P, 0, 2, 16, 32, P, P, P, None) == Q.QD_ERR_NULL
    assert r(P, 0, 2, 16, 32, P, None, None, None) == Q.QD_ERR_NULL
    assert r(P, 0, 1 << 31, 16, 32, P, P, None, None) == Q.QD_ERR_UNSUPPORTED
    assert r(None, 0, 0, 16, 32, None, None, None, None) == Q.QD_OK


def gemm(**kw):
    a = dict(a=P, s=P, a_rows=64, tok=P, offs=P, E=4, rows=64, w=P, ws=P, N=64, K=32, epi=0, out=P,
             os=P, wsp=P, n=BIG)
    a.update(kw)
    return Q.raw("moe_fp8_block_grouped_gemm", *a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(epi=3), Q.QD_ERR_DTYPE), (dict(E=0), Q.QD_ERR_SHAPE), (dict(rows=-1), Q.QD_ERR_SHAPE),
    (dict(K=24), Q.QD_ERR_SHAPE), (dict(K=0), Q.QD_ERR_SHAPE), (dict(N=12), Q.QD_ERR_SHAPE),
    (dict(N=96, epi=1), Q.QD_ERR_SHAPE), (dict(N=32, epi=2), Q.QD_ERR_SHAPE),
    (dict(offs=None), Q.QD_ERR_SHAPE), (dict(tok=None, rows=65), Q.QD_ERR_SHAPE),
    (dict(w=None), Q.QD_ERR_NULL), (dict(out=None), Q.QD_ERR_NULL),
    (dict(epi=2, os=None), Q.QD_ERR_NULL), (dict(a=P + 4), Q.QD_ERR_ALIGN),
    (dict(out=P + 8), Q.QD_ERR_ALIGN), (dict(tok=P + 2), Q.QD_ERR_ALIGN),
    (dict(epi=2, K=512, rows=8, wsp=None), Q.QD_ERR_WORKSPACE),
    (dict(epi=2, K=512, rows=8, n=64), Q.QD_ERR_WORKSPACE),
    (dict(epi=2, wsp=P + 8), Q.QD_ERR_ALIGN),
    (dict(E=1025), Q.QD_ERR_UNSUPPORTED), (dict(K=1 << 20, a_rows=4096), Q.QD_ERR_UNSUPPORTED),
    (dict(K=1 << 20, N=4096), Q.QD_ERR_UNSUPPORTED), (dict(rows=0, a=None, out=None), Q.QD_OK),
    (dict(rows=1 << 30), Q.QD_ERR_UNSUPPORTED), (dict(a_rows=1 << 30, rows=0), Q.QD_ERR_UNSUPPORTED),
])
def test_gemm_refusals(kw, want):
    assert gemm(**kw) == want


def test_gathered_rows_may_be_more_than_the_codes_hold(monkeypatch):
    """The 4 GiB are those of the activation codes, not of the rows that gather them: k
    rows of a long token each."""
    monkeypatch.setenv("QD_FAULT_INJECT", "launch")
    assert gemm(a_rows=1 << 16, rows=1 << 19, K=1 << 13) == Q.QD_ERR_HIP
    assert gemm(a_rows=1 << 19, rows=1 << 19, K=1 << 13) == Q.QD_ERR_UNSUPPORTED


def test_layer_refusals():
    n = Q.lib().qd_fp8_block_moe_layer_workspace(4, 64, 8, 2, 32)

    def call(**kw):
        a = dict(x=P, logits=P, T=4, H=64, E=8, k=2, I=32, scoring=0, bias=None, groups=1, top=1,
                 gsum=1, renorm=1, scale=1.0, live=None, w13=P, s13=P, w2=P, s2=P, y=P, ws=P, n=n)
        a.update(kw)
        return Q.raw("qd_fp8_block_moe_layer_forward", *a.values(), None)
    assert call(H=40) == Q.QD_ERR_SHAPE
    assert call(I=48) == Q.QD_ERR_SHAPE
    assert call(k=9) == Q.QD_ERR_SHAPE
    assert call(groups=3) == Q.QD_ERR_SHAPE
    assert call(scoring=7) == Q.QD_ERR_DTYPE
    assert call(n=n - 1) == Q.QD_ERR_WORKSPACE
    assert call(y=P + 8) == Q.QD_ERR_ALIGN
    assert call(w2=None) == Q.QD_ERR_NULL
    assert call(logits=None) == Q.QD_ERR_NULL


def test_wrappers_refuse_host_tensors():
    with pytest.raises(ValueError):
        ops.route_scored(torch.zeros(2, 8), 2)
    with pytest.raises(ValueError):
        ops.fp8_block_quantize_act(torch.zeros(2, 16))
    with pytest.raises(ValueError):
        ops.fp8_block_grouped_gemm(torch.zeros((2, 16), dtype=torch.uint8), None, None, None, 2)


def test_injected_launch_failure(monkeypatch):
    monkeypatch.setenv("QD_FAULT_INJECT", "launch")
    assert route() == Q.QD_ERR_HIP
    assert gemm() == Q.QD_ERR_HIP


def test_more_threads_than_a_launch_holds(monkeypatch):
    """One dimension of a launch has fewer than 2^32 threads: refused here, not by the launch."""
    monkeypatch.setenv("QD_FAULT_INJECT", "launch")
    huge = 1 << 45
    assert route(T=(1 << 26) - 4, n=huge) == Q.QD_ERR_HIP
    assert route(T=1 << 26, n=huge) == Q.QD_ERR_UNSUPPORTED
    back = lambda T: Q.raw("moe_route_scored_backward", P, 0, 16, T, 16, 2, 1, 1, 1.0, P, P, P, 16, None)
    assert back((1 << 26) - 4) == Q.QD_ERR_HIP and back(1 << 26) == Q.QD_ERR_UNSUPPORTED
    act = lambda rows: Q.raw("fp8_block_quantize_act", P, 0, rows, 16, 16, P, P, None)
    assert act((1 << 28) - 16) == Q.QD_ERR_HIP and act(1 << 28) == Q.QD_ERR_UNSUPPORTED
    bank = lambda groups: Q.raw("fp8_block_quantize_weight", P, 0, groups, 16, 16, P, P, None, None, None)
    assert bank((1 << 24) - 1) == Q.QD_ERR_HIP and bank(1 << 24) == Q.QD_ERR_UNSUPPORTED
    # the layer refuses before its first launch
    monkeypatch.delenv("QD_FAULT_INJECT")
    n = Q.lib().qd_fp8_block_moe_layer_workspace(1 << 26, 16, 16, 2, 32)
    assert Q.raw("qd_fp8_block_moe_layer_forward", P, P, 1 << 26, 16, 16, 2, 32, 0, None, 1, 1, 1, 1,
                 1.0, None, P, P, P, P, P, P, n, None) == Q.QD_ERR_UNSUPPORTED
