"""Attention over prompts and caches where it can go wrong: values that are no numbers, that overflow or are huge, sums that have a
closed form, arguments that do not fit, waits that run out."""
import numpy as np
import pytest
import torch

from oracle import cake_oracle as O
from paper_2503_12491_b200 import harness, synth
from paper_2503_12491_b200.binding import CAKE_ERR_ARG, CAKE_ERR_TIMEOUT
from test_gpu_attend import BF16, FP32, U, cached, check_cached, check_out, context, f64, prompt, run_cached, weight_error

pytestmark = pytest.mark.gpu
DTYPES = pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])


@DTYPES
@pytest.mark.parametrize("d", [64, 128])
def test_prompt_logits_that_are_no_numbers(dtype, d):
    """A row with a NaN among its logits has a log-sum-exp of NaN, not the -inf of a row without weight: a query that is NaN, and a
    first key that is (then row 0 sees nothing else, and the maximum of no logit of the first tile can be taken for a number)."""
    lens, sw = (300, 40), 16
    cake = context(4, 2, d, dtype, lens, window=sw)
    q, k, v = prompt(4, 2, d, dtype, lens, seed=6)
    good, good_lse = cake.attend_prompt(q, k, v)
    bad = torch.zeros(4, 340, dtype=torch.bool, device="cuda")
    q[:2, [0, 5, 200, 299], 3] = float("nan")
    bad[:2, [0, 5, 200, 299]] = True
    k[1, 300, 1] = float("nan")                       # the second request's first key, for heads 2 and 3
    bad[2:, 300:] = True
    q[1, 310] = float("nan")                          # every channel
    bad[1, 310] = True
    lw = torch.full((2, 4, sw), 7.0, device="cuda")
    out, lse = cake.attend_prompt(q, k, v, lse_window=lw)
    assert torch.equal(torch.isnan(lse), bad) and torch.isnan(out[bad]).all()
    assert torch.equal(lse[~bad], good_lse[~bad]) and torch.equal(out[~bad], good[~bad])
    want = torch.stack([lse[:, a - sw:a] for a in (300, 340)])
    assert torch.equal(torch.isnan(lw), torch.isnan(want)) and torch.equal(lw.nan_to_num(1.0), want.nan_to_num(1.0))


@DTYPES
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [1, 63, 64, 65, 130, 256])
def test_prompt_finite_inputs_whose_logits_overflow(dtype, d, bad):
    """Finite queries and keys with logits of -inf, also where the first tiles of a row have no other: they weigh nothing."""
    n = 300
    cake = context(2, 1, d, dtype, (n,))
    q, k, v = prompt(2, 1, d, dtype, (n,), seed=4)
    q[:, :, 0] = 2.0 ** 66
    k[:, :, 0] = 0
    k[:, :bad, 0] = -(2.0 ** 66)
    out, lse = cake.attend_prompt(q, k, v)
    assert torch.isnan(out[:, :bad]).all() and (lse[:, :bad] == float("-inf")).all()
    qn, kn, vn = f64(q[:, bad:]), f64(k[:, bad:]), f64(v[:, bad:])
    qn[:, :, 0] = 0                                   # (times a key's zero)
    check_out(f64(out[:, bad:]), f64(lse[:, bad:]), O.prompt_attention(qn, kn, vn), weight_error(qn, kn, d), n, dtype)


def huge(dtype, d, n, heads, size, seed):
    """Queries of +-size and keys 1..n in some order along one channel: logits size / sqrt(d) apart, of up to n times that."""
    g = torch.Generator().manual_seed(seed)
    sign = torch.where(torch.rand(heads, n, generator=g) < 0.5, -1.0, 1.0)
    order = torch.randperm(n, generator=g) + 1.0
    q, k = torch.zeros(heads, n, d), torch.zeros(1, n, d)
    q[:, :, 1], k[0, :, 1] = sign * size, order
    v = torch.randn(1, n, d, generator=g)
    return q.to(dtype).cuda(), k.to(dtype).cuda(), v.to(dtype).cuda(), sign.numpy(), order.numpy()


@DTYPES
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [2.0 ** 22, 2.0 ** 25, 2.0 ** 27, 2.0 ** 40, 2.0 ** 100], ids=lambda x: f"2^{int(np.log2(x))}")
def test_huge_logits(dtype, d, size):
    """Logits far beyond the 24 bits of fp32: all the weight is on the largest, and the output is its value.  Prompts, and the last
    queries over the same rows in a cache.  The cache's weight is 2^0 against a sum of 1: bit for bit.  The prompts' is p / p with
    some p: in bf16 the weight is rounded for its product and the output is rounded (2^-8 each); in fp32 six of nine products of
    p and v are taken (the others are below 2^-21 of it together), summed in steps cut at 2^-23 each, and divided (4 u)."""
    tol = 2.01 * 2.0 ** -8 if dtype == BF16 else 2.0 ** -21 + 6 * 2.0 ** -23 + 4 * U
    n, hq = 250, 4                                    # (keys are whole numbers of eight bits: exact in bf16)
    q, k, v, sign, order = huge(dtype, d, n, hq, size, seed=d)
    cake = context(hq, 1, d, dtype, (n,))
    out, lse = cake.attend_prompt(q, k, v)
    one, one_lse = cake.attend_cache(0, q[:, -1][None].contiguous(), k[0], v[0], torch.tensor([0, n], device="cuda"))
    on, vn = f64(out), f64(v)[0]
    for h in range(hq):
        for i in range(n):
            j = int(np.argmax(sign[h, i] * order[:i + 1]))
            top = sign[h, i] * order[j] * size / np.sqrt(d)
            assert (np.abs(on[h, i] - vn[j]) <= tol * np.abs(vn[j])).all(), (h, i)
            assert abs(float(lse[h, i]) - top) <= 6 * U * abs(top)
        assert torch.equal(one[0, h], v[0, j]) and abs(float(one_lse[0, h]) - top) <= 6 * U * abs(top)


# ------------------------------------------------------------------ accumulated attention from given log-sum-exps
@DTYPES
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (4, 1, 128)])
def test_accumulated_weights_of_one_are_counted_exactly(hq, hkv, d, dtype):
    """Logits and log-sum-exps of zero: every weight is 2^0 = 1, and a key's sum the number of queries behind it."""
    lens = (8, 135, 1, 700, 6, 7)
    cake = context(hq, hkv, d, dtype, lens)
    q, k, _ = prompt(hq, hkv, d, dtype, lens)
    got = cake.accumulate_attention(q.zero_(), k, torch.zeros(hq, sum(lens), device="cuda"))
    want = torch.cat([torch.arange(n, 0, -1, device="cuda") for n in lens]).float()
    assert torch.equal(got, want.expand(hkv, -1))


@DTYPES
def test_accumulated_weights_have_no_bias(dtype):
    """The last key of every request has one weight, exp(-lse) with logits of zero: against 64 bits.  A weight is off by at most
    2^-22 (two units in the last place of ex2.approx, more than the polynomial's 1.8e-7) and the rounding of its argument
    lse * log2(e), 2 u |lse| (the product's and the constant's).  All this is even around zero where lse is, and 1.3e-7 in the root
    mean square (the polynomial 0.64e-7, the product's third of 2 u |lse| log2(e), the constant's): the mean of the 750 weights
    of a column lies within 2e-8 at four standard deviations."""
    g = torch.Generator().manual_seed(0)
    lens = tuple(int(n) for n in torch.randint(1, 17, (3000,), generator=g))
    cake = context(2, 2, 64, dtype, lens)
    q, k, _ = prompt(2, 2, 64, dtype, lens)
    lse = ((torch.rand(2, sum(lens), generator=g) - 0.5) * 6).cuda()
    got = cake.accumulate_attention(q.zero_(), k, lse)
    last = np.cumsum(lens) - 1
    ln = f64(lse)[:, last]
    rel = f64(got)[:, last] * np.exp(ln) - 1
    assert (np.abs(rel) <= 2.0 ** -22 + 2 * U * np.abs(ln)).all(), np.abs(rel).max()
    for c in range(8):                                # (the units take the columns of a tile in turn)
        here = rel[:, (np.asarray(lens) - 1) % 8 == c]
        assert abs(here.mean()) <= 2e-8, (c, here.mean())


# ------------------------------------------------------------------ arguments
@DTYPES
def test_keys_and_values_of_a_cache_have_the_same_rows(dtype):
    """The offsets are those of both: values of another layer or an older compaction, with fewer rows, would be read past their end."""
    x = cached(4, 2, 64, dtype, (40, 3))
    cake = context(4, 2, 64, dtype, layers=2)
    want = run_cached(cake, x)
    for k, v in [(x["k"], x["v"][:-1]), (x["k"], x["v"][:5]), (x["k"][:-1], x["v"]), (x["k"], x["v"][:0])]:
        with pytest.raises(ValueError, match="v_cache: expected shape"):
            cake.attend_cache(1, x["q"], k, v, x["off"])
    assert all(torch.equal(a, b) for a, b in zip(run_cached(cake, x), want))


@DTYPES
def test_arguments_on_wrong_boundaries_are_refused(dtype):
    """Log-sum-exps, accumulated weights and offsets lie on boundaries of their elements, at any of them; pointers off these are
    refused before a launch."""
    lens, sw = (40, 33), 4
    cake = context(4, 2, 64, dtype, lens, window=sw, layers=2)
    lib, h, p = cake.lib, cake._h, lambda t, off=0: t.data_ptr() + off
    q, k, v = prompt(4, 2, 64, dtype, lens)
    want, want_lse = cake.attend_prompt(q, k, v)
    want_sum = cake.accumulate_attention(q, k, want_lse)
    out, lse = torch.empty_like(q), torch.zeros(4 * 73 + 1, device="cuda")
    lw, acc = torch.zeros(2 * 4 * sw + 1, device="cuda"), torch.zeros(2 * 73 + 1, device="cuda")
    heads, tokens = 73 * 64, 64

    def attend(lse_off, lw_off):
        return lib.cake_attend_prompt(h, p(q), heads, tokens, p(k), p(v), p(out), heads, tokens, p(lse, lse_off), p(lw, lw_off), None)

    def accumulate(lse_off, out_off):
        return lib.cake_accumulate_attention(h, p(q), heads, tokens, p(k), p(lse, lse_off), p(acc, out_off), None)

    assert [attend(2, 0), attend(1, 0), attend(0, 2), attend(0, 3), accumulate(2, 0), accumulate(0, 1)] == [CAKE_ERR_ARG] * 6
    torch.cuda.synchronize()
    assert attend(4, 4) == 0 and accumulate(4, 4) == 0
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse[1:].view(4, 73), want_lse) and torch.equal(acc[1:].view(2, 73), want_sum)
    assert torch.equal(lw[1:].view(2, 4, sw), torch.stack([want_lse[:, a - sw:a] for a in (40, 73)]))

    for group in (0, 32):
        x = cached(4, 2, 64, dtype, (40, 3), group=group, tail=(4, np.array([1, 2])))
        want, want_lse = run_cached(cake, x)
        need = lib.cake_attend_workspace_bytes(h, 2)
        ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty_like(want)
        lse, off = torch.zeros(9, device="cuda"), torch.cat([x["off"][:1], x["off"]])
        tl = torch.cat([x["tail"]["tail_len"][:1], x["tail"]["tail_len"]])
        c = x.get("cache")
        koff = torch.cat([c["kgroup_offsets"][:1], c["kgroup_offsets"]]) if group else None

        def call(o=8, t=4, l=4, g=8):
            tail = (p(x["tail"]["k_tail"]), p(x["tail"]["v_tail"]), p(tl, t), 4, p(out), p(lse, l), p(ws), need, None)
            if group:
                return lib.cake_attend_int4(h, 2, 1, p(x["q"]), p(c["k_codes"]), p(c["k_scale"]), p(c["k_zero"]), p(c["v_codes"]),
                                            p(c["v_scale"]), p(c["v_zero"]), group, p(off, o), p(koff, g), *tail)
            return lib.cake_attend_cache(h, 2, 1, p(x["q"]), p(x["k"]), p(x["v"]), p(off, o), *tail)

        assert [call(o=4), call(o=1), call(t=2), call(l=2), call(l=1)] == [CAKE_ERR_ARG] * 5
        assert not group or call(g=4) == CAKE_ERR_ARG
        torch.cuda.synchronize()
        assert call() == 0
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse[1:].view(2, 4), want_lse)


# ------------------------------------------------------------------ results handed from warp to warp
@pytest.mark.parametrize("group", [0, 32, 64])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 1)])
def test_short_ragged_fp32_requests_repeat_bit_for_bit(hq, hkv, group):
    """Most pairs end inside a CTA, where a warp puts together what the others left: always the same, and right."""
    rng = np.random.default_rng(hq + group)
    lens = tuple(int(n) for n in rng.choice([0, 1, 20, 33, 64, 65, 130, 260, 300, 390, 600], size=200))
    cake = context(hq, hkv, 64, FP32, layers=1)
    x = cached(hq, hkv, 64, FP32, lens, group=group, layers=1, layer=0, tail=(20, rng.integers(0, 21, size=200)))
    out, lse = check_cached(cake, x, FP32)
    for _ in range(40):
        again, lse2 = run_cached(cake, x)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    assert cake.status() == 0


# ------------------------------------------------------------------ waits that run out
@DTYPES
@pytest.mark.parametrize("d", [64, 128])
def test_waits_that_run_out_leave_the_context_usable(d, dtype):
    """A limit of one cycle.  (A wait on an mbarrier looks twice and sleeps for microseconds in between, so that short ones may still
    succeed: those of whole prompts in bf16 do not, nor those of warps for results of one another.)  Every kernel ends, after the
    copies and products that it has on their way, whatever the limit; the status says so; a call that reports nothing is right; and
    afterwards everything is as before."""
    lens, rows = (3000, 100), (60,) * 300
    cu = np.concatenate([[0], np.cumsum(lens)]).tolist()
    cake = context(8, 2, d, dtype, lens, layers=2)
    q, k, v = prompt(8, 2, d, dtype, lens)
    caches = [cached(8, 2, d, dtype, rows, group=g) for g in (0, 32)]
    lse = cake.attend_prompt(q, k, v)[1]
    calls = [lambda: cake.attend_prompt(q, k, v), lambda: (cake.accumulate_attention(q, k, lse),),
             lambda: run_cached(cake, caches[0]), lambda: run_cached(cake, caches[1])]
    good = [f() for f in calls]
    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))
    assert cake.status() == 0
    for i, f in enumerate(calls):
        ran_out = 0
        for _ in range(5):
            cake.begin(cu)
            cake.set_wait_limit(1)
            got = f()
            cake.set_wait_limit(0)
            status = cake.status()
            assert status in (0, CAKE_ERR_TIMEOUT)
            ran_out += status != 0
            assert status != 0 or same(got, good[i])
        assert ran_out or i == 1 or dtype == FP32
        cake.begin(cu)
        assert all(same(c(), w) for c, w in zip(calls, good)) and cake.status() == 0


# ------------------------------------------------------------------ decode caches
def test_a_decode_cache_before_and_after_its_first_step():
    """Before a layer's first step the free slots are rows of zeros, and attended; after it they hold the new token's rows."""
    d, hq, hkv, L, sw = 64, 4, 2, 2, 8
    w = synth.scaled(synth.workload(3), n_layers=L, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, seq_lens=(100, 60), total_budget=L * 30,
                     window=sw)
    qs, ks, vs = harness.device_inputs(w)
    cake = harness.cake_for(w)
    packed = cake.run(qs, ks, vs, w.cu_seqlens)
    kc, vc, off = cake.decode_begin(ks, vs)
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(2, h, d, generator=g).bfloat16().cuda() for h in (hq, hkv, hkv))
    o, p = off.cpu().numpy(), packed[2].cpu().numpy()

    def check(got, extra_k, extra_v):
        for r in range(2):
            n = (o[r * L + 1] - o[r * L]) // hkv
            assert (p[r * L + 1] - p[r * L]) // hkv == n - 1
            for h in range(hkv):
                rows = slice(p[r * L] + h * (n - 1), p[r * L] + (h + 1) * (n - 1))
                kn = np.concatenate([f64(packed[0][rows]), extra_k[r, h][None]])
                vn = np.concatenate([f64(packed[1][rows]), extra_v[r, h][None]])
                heads = slice(2 * h, 2 * h + 2)
                check_out(f64(got[0])[r, heads], f64(got[1])[r, heads], O.attend(f64(q)[r, heads], kn, vn),
                          weight_error(f64(q)[r, heads], kn, d), n, BF16)

    check(cake.attend_cache(0, q, kc, vc, off), np.zeros((2, hkv, d)), np.zeros((2, hkv, d)))
    cake.decode_step(0, q, k, v, kc, vc)
    check(cake.attend_cache(0, q, kc, vc, off), f64(k), f64(v))


# ------------------------------------------------------------------ beside the path
@DTYPES
def test_attention_on_a_stream_beside_the_eviction_path(dtype):
    """Scoring, eviction and compaction of a batch on one stream and all four attention calls of the same context on another, at the
    same time: each as by itself.  (The score kernel's CTAs wait for one another, and both sides hold tensor memory.)"""
    d, hq, hkv, L, sw = 128, 8, 2, 4, 16
    lens = (1700, 400)
    cu = [0, 1700, 2100]
    cake = context(hq, hkv, d, dtype, lens, window=sw, layers=L, budget=L * 80)
    layers = [prompt(hq, hkv, d, dtype, lens, seed=l) for l in range(L)]
    qw = [torch.stack([q[:, cu[r + 1] - sw:cu[r + 1]] for r in range(2)]).contiguous() for q, _, _ in layers]
    ks, vs = [x[1] for x in layers], [x[2] for x in layers]
    caches = [cached(hq, hkv, d, dtype, (900, 130, 33), group=g, layers=L) for g in (0, 32)]

    def path():
        cake.begin(cu)
        for l in range(L):
            cake.score_layer(l, qw[l], ks[l])
            cake.allocate(l)
            cake.evict(l)
        k, v, off, pos = cake.compact(ks, vs)
        return off, pos, k, v

    def attention():
        out, lse = cake.attend_prompt(*layers[0])
        return out, lse, cake.accumulate_attention(layers[0][0], ks[0], lse), *run_cached(cake, caches[0]), *run_cached(cake, caches[1])

    want, want_path = attention(), path()
    n = int(want_path[0][-1])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        with torch.cuda.stream(streams[0]):
            got_path = path()
        with torch.cuda.stream(streams[1]):
            for _ in range(6):
                got.append(attention())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
        assert torch.equal(got_path[0], want_path[0]) and all(torch.equal(a[:n], b[:n]) for a, b in zip(got_path[1:], want_path[1:]))
    assert cake.status() == 0
