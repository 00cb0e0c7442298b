"""Tight bounds on attention, at inputs whose sums are short: what the fp32 kernels' three bf16 terms per number and the bf16 kernels' two
per weight are there for.  u = 2^-24.

fp32 prompts.  A number is x1 + x2 + x3, cut after 8 and 16 bits: x2 below 2^-7 of it and x3 below 2^-15.  Of the nine products x2 y3
and x3 y2 (2^-22 each) and x3 y3 are not taken; the sum of six is cut at 2^-23 of itself at each step, once per product where
one channel or key alone is not zero.  Together CUT = 2 * 2^-22 + 2^-30 + 6 * 2^-23 of |x y|, 20 u.  A third term that is lost, or
multiplied with the wrong one, is up to 2^-15 of a product off: 512 u.
"""
import numpy as np
import pytest
import torch

from oracle import cake_oracle as O
from test_gpu_attend import BF16, FP32, U, cached, context, f64, prompt, run_cached

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


# ------------------------------------------------------------------ bf16: weights in two terms
def bf16_cut(x):
    """The upper 16 bits of x in fp32: one bf16 term of a weight."""
    return (np.asarray(x, np.float32).view(np.uint32) & 0xFFFF0000).view(np.float32).astype(np.float64)


def logits_of_one_channel(R, N, hq, hkv, d, rng):
    """Queries of a power of two or 1.5 of one along one channel, all heads alike, and keys there of whole eighths between -1 and 7/8:
    logits without any rounding but the scale's, and their weights."""
    q = np.zeros((R, hq, d))
    q[:, :, 5] = rng.choice([-3.0, -2.0, 2.0, 3.0], size=(R, 1))
    code = rng.integers(0, 16, size=(R, hkv, N))
    s = q[:, :hkv, 5][..., None] * (code - 8) / 8 / np.sqrt(d)
    p = np.exp(s)
    return q, code, p / p.sum(-1, keepdims=True)


@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (6, 2, 64), (2, 2, 128)])
@pytest.mark.parametrize("N,tail", [(2, 0), (33, 0), (100, 0), (300, 9), (1, 1)])
def test_bf16_rows_have_weights_in_two_terms(hq, hkv, d, N, tail):
    """Up to four query heads on a KV head.  The last value of every head makes the output vanish but for its own rounding, so that
    the output's rounding does not hide that of the weights: 2^-16 of the spread for two bf16 terms (the first cut, 2^-7, the rest
    rounded to 2^-9 of it), 6 u for the logit's scale and the exponential, u per addition of a sum.  One term, cut, is far off."""
    rng = np.random.default_rng(N + d)
    R, M = 8, N + tail
    q, code, p = logits_of_one_channel(R, M, hq, hkv, d, rng)
    k = np.zeros((R, hkv, M, d))
    k[..., 5] = (code - 8) / 8
    v = torch.tensor(rng.normal(size=(R, hkv, M, d))).bfloat16().double().numpy()
    v[:, :, -1] = torch.tensor(-(p[..., :-1, None] * v[:, :, :-1]).sum(2) / p[:, :, -1:]).bfloat16().double().numpy()
    want, spread = ((p[..., None] * x).sum(2) for x in (v, np.abs(v)))
    lim = (2.0 ** -16 + (6 + M) * U) * spread + 2.0 ** -8 * np.abs(want) + 1e-30
    top = p / p.max(-1, keepdims=True)
    once = (bf16_cut(top)[..., None] * v).sum(2) / top.sum(-1)[..., None]
    assert (np.abs(once - want) > 4 * lim).mean() > 0.2
    dev = lambda x: torch.tensor(x).bfloat16().cuda().contiguous()
    rows = lambda x, lo, hi: dev(x[:, :, lo:hi].reshape(-1, d))
    off = torch.arange(0, R + 1, device="cuda") * (hkv * N)
    kw = {}
    if tail:
        kw = dict(k_tail=dev(k[:, :, N:]), v_tail=dev(v[:, :, N:]), tail_len=torch.full((R,), tail, dtype=torch.int32, device="cuda"))
    out, _ = context(hq, hkv, d, BF16).attend_cache(0, dev(q), rows(k, 0, N), rows(v, 0, N), off, **kw)
    got = f64(out).reshape(R, hkv, hq // hkv, d)
    bad = np.abs(got - want[:, :, None]) / lim[:, :, None]
    assert (bad <= 1).all(), bad.max()


@pytest.mark.parametrize("hq,hkv,d,group", [(4, 1, 128, 32), (8, 1, 128, 32), (8, 1, 64, 64), (2, 2, 64, 32), (4, 2, 128, 128),
                                            (4, 1, 128, 64)])
@pytest.mark.parametrize("N", [2, 34, 100])
def test_4_bit_values_have_weights_times_scales_in_two_terms(hq, hkv, d, group, N):
    """Values scale * (code - 8), two rows after another of which cancel: their codes less 8 are 6 and -4 (3 and -2), the second's scale
    the first's times 3/2 and the ratio of their weights.  What is left: 2^-16 of the spread for two bf16 terms of weight times
    scale (as above), 6 u for the logit's scale and the exponential, 2 u for the scale and its product with the weight, u per addition.  One
    term is far off."""
    rng = np.random.default_rng(N + d + hq)
    R, ng = 4, d // group
    q, code, p = logits_of_one_channel(R, N, hq, hkv, d, rng)
    kc = rng.integers(0, 16, size=(R, hkv, N, d)).astype(np.uint8)           # (other channels meet queries of zero)
    kc[..., 5] = code
    scale = np.exp(rng.normal(size=(R, hkv, N, ng)))
    scale[:, :, 1::2] = scale[:, :, 0::2] * 1.5 * (p[:, :, 0::2] / p[:, :, 1::2])[..., None]
    scale = scale.astype(np.float32)
    a = rng.choice([6, 3, -6, -3], size=(R, hkv, N // 2, d)) * 1
    vc = np.empty((R, hkv, N, d), np.uint8)
    vc[:, :, 0::2], vc[:, :, 1::2] = 8 + a, 8 - a * 2 // 3
    per = np.repeat(scale.astype(np.float64), group, -1) * (vc.astype(np.float64) - 8)
    want, spread = ((p[..., None] * x).sum(2) for x in (per, np.abs(per)))
    lim = (2.0 ** -16 + (8 + N) * U) * spread + 2.0 ** -8 * np.abs(want) + 1e-30
    top = (p / p.max(-1, keepdims=True)).astype(np.float32)
    x = bf16_cut(top[..., None] * scale)
    once = (np.repeat(x, group, -1) * (vc.astype(np.float64) - 8)).sum(2) / top.sum(-1, dtype=np.float64)[..., None]
    assert (np.abs(once - want) > 4 * lim).mean() > 0.2
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    groups = R * hkv * -(-N // group)
    cache = dict(k_codes=dev(O.pack_nibbles(kc.reshape(-1, d))), k_scale=dev(np.full((groups, d), 0.125, np.float32)),
                 k_zero=dev(np.full((groups, d), -1.0, np.float32)), v_codes=dev(O.pack_nibbles(vc.reshape(-1, d))),
                 v_scale=dev(scale.reshape(-1, ng)), v_zero=dev((-8 * scale).reshape(-1, ng)),
                 row_offsets=torch.arange(0, R + 1, device="cuda") * (hkv * N),
                 kgroup_offsets=torch.arange(0, R + 1, device="cuda") * (hkv * -(-N // group)))
    out, _ = context(hq, hkv, d, BF16).attend_int4(0, torch.tensor(q).bfloat16().cuda(), cache)
    got = f64(out).reshape(R, hkv, hq // hkv, d)
    bad = np.abs(got - want[:, :, None]) / lim[:, :, None]
    assert (bad <= 1).all(), bad.max()
