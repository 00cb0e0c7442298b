"""Tight bounds on attention, at inputs whose sums are short: what the fp32 kernels' three bf16 terms per number are there for.
u = 2^-24.

fp32 prompts.  A number is x1 + x2 + x3, cut after 8 and 16 bits: x2 below 2^-7 of it and x3 below 2^-15.  Of the nine products x2 y3
and x3 y2 (2^-22 each) and x3 y3 are not taken; the sum of six is cut at 2^-23 of itself at each step, once per product where
one channel or key alone is not zero.  Together CUT = 2 * 2^-22 + 2^-30 + 6 * 2^-23 of |x y|, 20 u.  A third term that is lost, or
multiplied with the wrong one, is up to 2^-15 of a product off: 512 u.
"""
import numpy as np
import pytest
import torch

from oracle import cake_oracle as O
from test_gpu_attend import FP32, U, cached, context, f64, prompt, run_cached

pytestmark = pytest.mark.gpu
CUT = 2 * 2.0 ** -22 + 2.0 ** -30 + 6 * 2.0 ** -23


def one_channel(hq, hkv, d, n_req, length, g, size=1.0):
    """Requests of `length` tokens; request r's queries and keys have one channel that is not zero, another one than its neighbours'."""
    T = n_req * length
    q, k = torch.zeros(hq, T, d), torch.zeros(hkv, T, d)
    at = (torch.arange(T) // length) % d
    q[:, torch.arange(T), at] = torch.randn(hq, T, generator=g) * size
    k[:, torch.arange(T), at] = torch.randn(hkv, T, generator=g) * size
    return q.cuda(), k.cuda(), torch.randn(hkv, T, d, generator=g).cuda()


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (4, 1, 128), (3, 3, 128)])
def test_fp32_logits_and_values_of_single_tokens(hq, hkv, d):
    """Requests of one token: its log-sum-exp is its logit (CUT; the scale, the reference, ln 2 and their products, 8 u), its output its
    value (CUT of p v, and the sum of p, its inverse and the product, 4 u), its accumulated weight with log-sum-exps of zero
    exp(logit) (the logit's error, u |logit| twice for the exponent's argument, ex2.approx 4 u, the mean 4 u)."""
    g = torch.Generator().manual_seed(d + hq)
    R = 6 * d
    q, k, v = one_channel(hq, hkv, d, R, 1, g, size=2.0)
    cake = context(hq, hkv, d, FP32, (1,) * R)
    out, lse = cake.attend_prompt(q, k, v)
    acc = cake.accumulate_attention(q, k, torch.zeros_like(lse))
    G = hq // hkv
    kn, vn = (np.repeat(f64(x), G, 0) for x in (k, v))
    s = (f64(q) * kn).sum(-1) / np.sqrt(d)
    assert (np.abs(f64(lse) - s) <= (CUT + 8 * U) * np.abs(s)).all()
    assert (np.abs(f64(out) - vn) <= (CUT + 4 * U) * np.abs(vn)).all()
    e = np.exp(s)
    want, lim = (x.reshape(hkv, G, R).mean(1) for x in (e, e * ((CUT + 10 * U) * np.abs(s) + 8 * U)))
    assert (np.abs(f64(acc) - want) <= lim).all(), (np.abs(f64(acc) - want) / lim).max()


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (4, 1, 128)])
def test_fp32_weights_times_values_of_two_tokens(hq, hkv, d):
    """The second row of requests of two tokens: its weights have all three terms.  A weight is off by its logit's error, relative
    (CUT + 8 u of |logit|, for both logits), 4 u of its exponential and u of its sum; products and their sum by CUT."""
    g = torch.Generator().manual_seed(d)
    R = 4 * d
    q, k, v = one_channel(hq, hkv, d, R, 2, g)
    out, _ = context(hq, hkv, d, FP32, (2,) * R).attend_prompt(q, k, v)
    G = hq // hkv
    pair = lambda x: np.repeat(f64(x), G, 0).reshape(hq, R, 2, d)
    kn, vn = pair(k), pair(v)
    qn, got = f64(q).reshape(hq, R, 2, d)[:, :, 1], f64(out).reshape(hq, R, 2, d)[:, :, 1]
    s = (qn[:, :, None] * kn).sum(-1) / np.sqrt(d)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    want, spread = (p[..., None] * vn).sum(2), (p[..., None] * np.abs(vn)).sum(2)
    lim = (2 * (CUT + 8 * U) * np.abs(s).max(-1)[..., None] + CUT + 9 * U) * spread + 4 * U * np.abs(want)
    assert (np.abs(got - want) <= lim).all(), (np.abs(got - want) / lim).max()


def norm(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [512, 1500])
def test_fp32_prompts_in_the_norm(d, n):
    """Errors that are not alike add up like values do: in the norm an output is as far off as a typical weight of it, relative.  A
    logit of size 2 and a bit is cut at 2^-24 of its partial sums in d / 16 steps of the leading product, on average: up to
    8 * 2^-24 * 2 = 1e-6, less what the first steps' smaller sums and the size of a typical logit (half of it below 1.4) take off;
    the sums of weights times values, 64 keys at a time, four steps: 2e-7.  So 1e-6 is never reached; with two terms per number
    it is 2e-5, and with outputs summed over the keys in tensor memory 2e-6 at 512 keys.  Accumulated weights lose less: what logits
    lose their log-sum-exps have lost too."""
    cake = context(4, 2, d, FP32, (n,))
    q, k, v = prompt(4, 2, d, FP32, (n,), seed=n + d)
    out, lse = cake.attend_prompt(q, k, v)
    qn, kn, vn = f64(q), f64(k), f64(v)
    want, want_lse, _ = O.prompt_attention(qn, kn, vn)
    assert norm(f64(out), want) <= 1e-6
    assert norm(f64(lse), want_lse) <= 1e-6
    assert norm(f64(cake.accumulate_attention(q, k, lse)), O.cumulative_attention(qn, kn)) <= 1e-6


@pytest.mark.parametrize("group", [0, 32])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (8, 1, 128)])
def test_fp32_caches_in_the_norm(hq, hkv, d, group):
    """fp32 FMA throughout: a logit's d roundings of its partial sums, u / 2 each and not alike, are (d / 2)^1/2 u / 2 of a logit of size
    2 to 4, at most 1e-6 for 128 channels; in the norm of the outputs less by the spread of the weights, as above."""
    lens = (700, 90, 1500)
    x = cached(hq, hkv, d, FP32, lens, group=group, layers=1, layer=0)
    out, _ = run_cached(context(hq, hkv, d, FP32), x)
    qn, on = f64(x["q"]), f64(out)
    want = np.zeros_like(on)
    for r, n in enumerate(lens):
        for h in range(hq):
            rows = slice(x["offn"][r] + (h * hkv // hq) * n, x["offn"][r] + (h * hkv // hq + 1) * n)
            want[r, h] = O.attend(qn[r, h:h + 1], x["kn"][rows], x["vn"][rows])[0][0]
    assert norm(on, want) <= 1e-6
