"""Attention over prompts and caches against the oracle in 64 bits.

Bounds.  u = 2^-24 is half a step of fp32.  A logit is a dot product of d terms, each rounded, summed in fp32 (up to a whole
step per addition on the tensor cores) and scaled: it is off by at most ds = (2 d + 16) u E with E = sum_c |q_c k_c| / sqrt(d),
the largest over the visible keys; the exponential adds 4 u, relative, and the reduction of its argument 2 u times the
logits' range, which is at most 2 E.  A weight is therefore off by dw = (2 d + 20) u E + 4 u, relative, and a sum of N of them by
dw + N u.  An output is a weighted mean: off by (2 dw + 2 N u) S with S = sum_j p_j |v_j|.  bf16: the weights are rounded
to 2^-8, relative, before they are multiplied with the values (2^-8 S more), and the output is rounded to 2^-8 of itself.
4-bit keys under bf16 queries: the products q * scale are held in two bf16 terms, 2^-16 relative.
"""
import numpy as np
import pytest
import torch

from oracle import cake_oracle as O
from paper_2503_12491_b200 import Cake, CakeError, binding, synth, harness
from paper_2503_12491_b200.binding import CAKE_ERR_ARG, CAKE_ERR_STATE

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, FP32 = torch.bfloat16, torch.float32


def f64(t):
    return t.detach().double().cpu().numpy()


def context(hq, hkv, d, dtype, lens=(), window=1, layers=1, budget=None, **kw):
    cake = Cake(n_layers=layers, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, window=window, pool_kernel=1, gamma=200.0,
                total_budget=budget or layers * max(window, 64), max_requests=max(1, len(lens)),
                max_total_tokens=max(1, sum(lens)), dtype=dtype, **kw)
    if lens:
        cake.begin(np.concatenate([[0], np.cumsum(lens)]).tolist())
    return cake


def weight_error(q, k, d):
    """dw of the module's docstring; q, k as the magnitudes that enter the products."""
    E = np.abs(q).max() * np.abs(k).max() * np.sqrt(d)         # bounds sum_c |q_c k_c| / sqrt(d)
    E = min(E, np.sqrt((q ** 2).sum(-1).max() * (k ** 2).sum(-1).max() / d))
    return (2 * d + 20) * U * E + 4 * U


def check_out(got, lse, want, dw, n, dtype, extra=0.0):
    out, ref_lse, spread = want
    rel = 2 * dw + 2 * n * U + (2.0 ** -8 if dtype == BF16 else 0.0) + extra
    tol = rel * spread + (2.0 ** -8 if dtype == BF16 else U) * np.abs(out) + 1e-30
    assert np.isfinite(got).all() or not np.isfinite(out).all()
    bad = ~(np.abs(got - out) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], out[bad][:4], tol[bad][:4])
    if lse is not None:
        fin = np.isfinite(ref_lse)
        assert np.array_equal(lse[~fin], ref_lse[~fin])
        lim = 2 * dw + n * U + 4 * U * np.abs(ref_lse[fin])
        assert (np.abs(lse[fin] - ref_lse[fin]) <= lim).all(), (np.abs(lse[fin] - ref_lse[fin]) / lim).max()


def prompt(hq, hkv, d, dtype, lens, seed=0, layout="heads", temperature=2.0):
    g = torch.Generator().manual_seed(seed)
    T = sum(lens)
    q = (torch.randn(hq, T, d, generator=g) * temperature).to(dtype)
    k, v = torch.randn(hkv, T, d, generator=g).to(dtype), torch.randn(hkv, T, d, generator=g).to(dtype)
    k[:, ::37] *= 3
    q, k, v = (x.cuda() for x in (q, k, v))
    if layout == "tokens":
        q = q.transpose(0, 1).contiguous().transpose(0, 1)
    elif layout == "fused":                          # a slice of a fused projection's output: [T][H_q + 2 H_kv][d]
        buf = torch.full((T, hq + 2 * hkv, d), float("nan"), dtype=dtype, device="cuda")
        buf[:, :hq] = q.transpose(0, 1)
        q = buf[:, :hq].transpose(0, 1)
    return q, k, v


def check_prompt(cake, q, k, v, lens, dtype, window=1, **kw):
    hq, T, d = q.shape
    lw = torch.full((len(lens), hq, window), 7.0, device="cuda")
    out, lse = cake.attend_prompt(q, k, v, lse_window=lw, **kw)
    received = cake.accumulate_attention(q, k, lse)
    assert out.dtype == dtype and out.shape == q.shape and cake.status() == 0
    qn, kn, vn, on, ln, rn = (f64(x) for x in (q, k, v, out, lse, received))
    a = 0
    for r, n in enumerate(lens):
        s = slice(a, a + n)
        dw = weight_error(qn[:, s], kn[:, s], d)
        want = O.prompt_attention(qn[:, s], kn[:, s], vn[:, s])
        check_out(on[:, s], ln[:, s], want, dw, n, dtype)
        assert torch.equal(lw[r], lse[:, a + n - window:a + n])
        # given the device's lse (fp32), a weight is off by dw and the rounding of the exponent's terms
        ref = O.cumulative_attention(qn[:, s], kn[:, s])
        lim = (4 * dw + 4 * U * np.abs(want[1]).max() + (hq // k.shape[0] + 4) * n * U) * ref + 1e-30
        assert (np.abs(rn[:, s] - ref) <= lim).all(), (np.abs(rn[:, s] - ref) / lim).max()
        a += n
    return out, lse, received


HEADS = [(4, 4, 64), (8, 2, 128), (8, 1, 64), (3, 3, 128), (4, 2, 64), (6, 2, 128)]
LENS = [(1,), (2, 1, 5), (63, 64, 65), (127, 128, 129), (200, 1, 31), (255, 256, 257), (385, 511), (700,)]


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_prompt_lengths(dtype, lens):
    cake = context(4, 2, 128, dtype, lens)
    check_prompt(cake, *prompt(4, 2, 128, dtype, lens, seed=len(lens)), lens, dtype)


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["heads", "tokens", "fused"])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_prompt_heads_and_layouts(hq, hkv, d, layout, dtype):
    lens = (150, 33, 290)
    cake = context(hq, hkv, d, dtype, lens, window=16)
    check_prompt(cake, *prompt(hq, hkv, d, dtype, lens, seed=hq, layout=layout), lens, dtype, window=16)


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
def test_prompt_many_requests(dtype):
    """More requests than one launch takes."""
    rng = np.random.default_rng(3)
    lens = tuple(int(x) for x in rng.integers(1, 40, size=300))
    cake = context(2, 1, 64, dtype, lens)
    check_prompt(cake, *prompt(2, 1, 64, dtype, lens), lens, dtype)


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("temperature", [0.0, 30.0])
def test_prompt_flat_and_sharp_attention(dtype, temperature):
    """All weights equal, and logits far apart (the running reference moves often)."""
    lens = (333, 130)
    cake = context(4, 2, 64, dtype, lens)
    q, k, v = prompt(4, 2, 64, dtype, lens, temperature=temperature)
    k[:, 200:] *= 2                                   # the largest logits come late
    check_prompt(cake, q, k, v, lens, dtype)


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_prompt_what_lies_behind_has_no_influence(dtype, d, bad):
    lens = (130, 70, 300)
    cake = context(4, 2, d, dtype, lens)
    q, k, v = prompt(4, 2, d, dtype, lens)
    good = cake.attend_prompt(q, k, v)
    good_sum = cake.accumulate_attention(q, k, good[1])
    k2, v2, q2 = k.clone(), v.clone(), q.clone()
    at = 200 + 140                                    # token 140 of the third request
    k2[:, 130:200] = bad; v2[:, 130:200] = bad; q2[:, 130:200] = bad      # the whole second request
    k2[:, at] = bad; v2[:, at] = bad
    out, lse = cake.attend_prompt(q2, k2, v2)
    for s in (slice(0, 130), slice(200, at)):
        assert torch.equal(out[:, s], good[0][:, s]) and torch.equal(lse[:, s], good[1][:, s])
    # the rows that do see it: NaN if its key is not a number, or wherever its value is not finite
    assert not torch.isfinite(out[:, at:]).any()
    # only the value is bad: every row from there on has it
    v3 = v.clone()
    v3[0, at] = bad
    out = cake.attend_prompt(q, k, v3)[0]
    assert torch.equal(out[:, :at], good[0][:, :at]) and torch.equal(out[2:], good[0][2:])
    assert not torch.isfinite(out[:2, at:]).any()
    lse2 = good[1].clone()
    lse2[:, 130:200] = bad
    got = cake.accumulate_attention(q2[:, :], k, lse2)
    for s in (slice(0, 130), slice(200, 500)):
        assert torch.equal(got[:, s], good_sum[:, s])


def test_prompt_outputs_given_and_rows_around_them():
    """Outputs into the caller's strided buffer: nothing beside the rows is written."""
    lens = (129, 40)
    T = sum(lens)
    cake = context(4, 2, 128, BF16, lens, window=8)
    q, k, v = prompt(4, 2, 128, BF16, lens, layout="tokens")
    buf = torch.full((T + 4, 6, 128), 5.0, dtype=BF16, device="cuda")
    lse = torch.full((4, T), 3.0, device="cuda")
    out, lse2 = cake.attend_prompt(q, k, v, out=buf[2:T + 2, 1:5].transpose(0, 1), lse=lse)
    assert out.data_ptr() == buf[2, 1].data_ptr() and lse2.data_ptr() == lse.data_ptr()
    want, want_lse = cake.attend_prompt(q, k, v)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert (buf[:2] == 5).all() and (buf[T + 2:] == 5).all() and (buf[:, 0] == 5).all() and (buf[:, 5] == 5).all()


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
def test_prompt_repeats_bit_for_bit_on_streams_and_in_graphs(dtype):
    lens = (900, 77)
    cake = context(8, 2, 128, dtype, lens)
    q, k, v = prompt(8, 2, 128, dtype, lens)
    out, lse = cake.attend_prompt(q, k, v)
    got = cake.accumulate_attention(q, k, lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o2, l2 = cake.attend_prompt(q, k, v)
        g2 = cake.accumulate_attention(q, k, l2)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, o2) and torch.equal(lse, l2) and torch.equal(got, g2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o3, l3 = cake.attend_prompt(q, k, v)
        g3 = cake.accumulate_attention(q, k, l3)
    cake.begin([0, 5])                                # the graph does not depend on the context's batch
    q.mul_(0.5)
    graph.replay()
    cake.begin([0, 900, 977])
    o4, l4 = cake.attend_prompt(q, k, v)
    assert torch.equal(o3, o4) and torch.equal(l3, l4) and torch.equal(g3, cake.accumulate_attention(q, k, l4))


def test_prompt_refusals():
    cake = context(4, 2, 64, BF16)
    q, k, v = prompt(4, 2, 64, BF16, (40,))
    with pytest.raises((CakeError, ValueError)):     # no batch
        cake.attend_prompt(q, k, v)
    cake = context(4, 2, 64, BF16, (40,))
    cake.attend_prompt(q, k, v)
    for bad in [(q.float(), k, v), (q[:2], k, v), (q, k[:, :39], v), (q, k, v.transpose(0, 1)), (q.cpu(), k, v),
                (q.transpose(1, 2), k, v), (q, k.float(), v)]:
        with pytest.raises(ValueError):
            cake.attend_prompt(*bad)
    flat = torch.zeros(4 * 40 * 64 + 64, dtype=BF16, device="cuda")
    odd = flat[1:1 + 4 * 40 * 64].view(4, 40, 64)    # not on a 16-byte boundary
    with pytest.raises(CakeError) as e:
        cake.attend_prompt(odd, k, v)
    assert e.value.code == CAKE_ERR_ARG
    strided = torch.zeros(4, 40, 68, dtype=BF16, device="cuda")[:, :, :64]      # rows 136 bytes apart
    with pytest.raises(CakeError):
        cake.attend_prompt(strided, k, v)
    with pytest.raises(CakeError):                   # rows of the output overlap
        cake.attend_prompt(q, k, v, out=flat[:64].as_strided((4, 40, 64), (0, 64, 1)))
    with pytest.raises(CakeError):
        cake.attend_prompt(q, k, v, out=flat.as_strided((4, 40, 64), (64, 64, 1)))
    with pytest.raises(ValueError):
        cake.accumulate_attention(q, k, torch.zeros(4, 39, device="cuda"))
    empty = context(4, 2, 64, BF16)
    empty.begin([0])
    out, lse = empty.attend_prompt(q[:, :0], k[:, :0], v[:, :0])
    assert out.shape == (4, 0, 64) and lse.shape == (4, 0)


def test_one_query_tensor_for_all_heads():
    """Strides of zero between heads are fine for what is only read."""
    lens = (70,)
    cake = context(4, 2, 64, BF16, lens)
    q, k, v = prompt(1, 2, 64, BF16, lens)[0], *prompt(4, 2, 64, BF16, lens)[1:]
    a = cake.attend_prompt(q.expand(4, 70, 64), k, v)
    b = cake.attend_prompt(q.expand(4, 70, 64).contiguous(), k, v)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------ caches
def cached(hq, hkv, d, dtype, lens, group=0, tail=None, layers=2, layer=1, seed=0):
    """A packed cache of `layers` layers whose `layer` has lens[r] rows per head; its rows in float64 for the oracle."""
    g = torch.Generator().manual_seed(seed)
    R = len(lens)
    block = [lens[r] if l == layer else (3 * r + l) % 5 for r in range(R) for l in range(layers)]
    off = np.concatenate([[0], np.cumsum([hkv * n for n in block])])
    rows = int(off[-1])
    spare = 3                                         # rows behind the last block: never read
    k, v = torch.randn(rows, d, generator=g), torch.randn(rows, d, generator=g)
    k[::11] *= 3
    k, v = k.to(dtype), v.to(dtype)
    q = (torch.randn(R, hq, d, generator=g) * 2).to(dtype)
    x = dict(q=q.cuda(), off=torch.tensor(off, dtype=torch.int64, device="cuda"), tail={})
    kn, vn, mag = f64(k), f64(v), None
    if group:
        koff = np.concatenate([[0], np.cumsum([hkv * -(-n // group) for n in block])])
        kc, vc = np.zeros((rows, d), np.uint8), np.zeros((rows, d), np.uint8)
        ks, kz = np.zeros((max(int(koff[-1]), 1), d), np.float32), np.zeros((max(int(koff[-1]), 1), d), np.float32)
        vc, vs, vz = O.quantize_values_per_token(v.float().numpy(), group)
        vn, mag = O.dequantize_values(vc, vs, vz, group), np.zeros((rows, d))
        kn = np.zeros((rows, d))
        for i, n in enumerate(block):
            for h in range(hkv if n else 0):
                a, ga, gn = off[i] + h * n, koff[i] + h * -(-n // group), -(-n // group)
                c, s, z = O.quantize_keys_per_channel(k[a:a + n].float().numpy(), group)
                kc[a:a + n], ks[ga:ga + gn], kz[ga:ga + gn] = c, s, z
                kn[a:a + n] = O.dequantize_keys(c, s, z, group)
                mag[a:a + n] = np.repeat(np.abs(z) + 15 * s, group, 0)[:n]
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        pad = lambda a: np.concatenate([a, np.full((spare,) + a.shape[1:], 255 if a.dtype == np.uint8 else np.nan, a.dtype)])
        x["cache"] = dict(k_codes=dev(pad(O.pack_nibbles(kc))), k_scale=dev(pad(ks)), k_zero=dev(pad(kz)),
                          v_codes=dev(pad(O.pack_nibbles(vc))), v_scale=dev(pad(vs)), v_zero=dev(pad(vz)),
                          row_offsets=x["off"], kgroup_offsets=torch.tensor(koff, dtype=torch.int64, device="cuda"))
    else:
        nan = torch.full((spare, d), float("nan"), dtype=dtype)
        x["k"], x["v"] = torch.cat([k, nan]).cuda(), torch.cat([v, nan]).cuda()
    if tail is not None:
        cap, tl = tail
        kt, vt = torch.randn(R, hkv, cap, d, generator=g).to(dtype), torch.randn(R, hkv, cap, d, generator=g).to(dtype)
        x["tail_rows"] = (f64(kt), f64(vt), np.clip(tl, 0, cap))
        for r in range(R):
            n = int(x["tail_rows"][2][r])
            kt[r, :, n:], vt[r, :, n:] = float("nan"), float("inf")
        x["tail"] = dict(k_tail=kt.cuda(), v_tail=vt.cuda(), tail_len=torch.tensor(tl, dtype=torch.int32, device="cuda"))
    x.update(kn=kn, vn=vn, mag=mag, offn=off, lens=lens, layers=layers, layer=layer, group=group)
    return x


def run_cached(cake, x, **kw):
    if x["group"]:
        return cake.attend_int4(x["layer"], x["q"], x["cache"], **x["tail"], **kw)
    return cake.attend_cache(x["layer"], x["q"], x["k"], x["v"], x["off"], **x["tail"], **kw)


def check_cached(cake, x, dtype):
    out, lse = run_cached(cake, x)
    R, hq, d = x["q"].shape
    hkv = cake.cfg.n_kv_heads
    on, ln, qn = f64(out), f64(lse), f64(x["q"])
    for r, n in enumerate(x["lens"]):
        for g in range(hkv):
            a = x["offn"][r * x["layers"] + x["layer"]] + g * n
            k, v = x["kn"][a:a + n], x["vn"][a:a + n]
            mag = np.abs(k) if x["mag"] is None else x["mag"][a:a + n]
            if "tail_rows" in x:
                t = x["tail_rows"][2][r]
                kt, vt = x["tail_rows"][0][r, g, :t], x["tail_rows"][1][r, g, :t]
                k, v, mag = np.concatenate([k, kt]), np.concatenate([v, vt]), np.concatenate([mag, np.abs(kt)])
            heads = slice(g * (hq // hkv), (g + 1) * (hq // hkv))
            want = O.attend(qn[r, heads], k, v)
            if len(k) == 0:
                assert (on[r, heads] == 0).all() and (ln[r, heads] == -np.inf).all()
                continue
            dw = weight_error(qn[r, heads], mag, d)
            if x["group"]:
                E = np.sqrt((qn[r, heads] ** 2).sum(-1).max() * (mag ** 2).sum(-1).max() / d)
                dw += (2.0 ** -16 if dtype == BF16 else 4 * U) * E
                # values: zero + code * scale, each product rounded: the spread counts their magnitudes
                vm = np.abs(v).max()
                want = (want[0], want[1], np.maximum(want[2], 2 * vm))
            check_out(on[r, heads], ln[r, heads], want, dw, len(k), dtype)
    return out, lse


CACHE_LENS = [(1,), (0, 3), (15, 16, 17), (31, 32, 33, 0), (63, 64, 65), (127, 130, 1), (500, 7), (1500,)]


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("lens", CACHE_LENS, ids=str)
def test_cache_lengths(dtype, group, lens):
    cake = context(8, 2, 128, dtype, layers=2)
    check_cached(cake, cached(8, 2, 128, dtype, lens, group, seed=sum(lens)), dtype)


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("group", [0, 32, 64])
@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 64), (8, 1, 128), (8, 1, 64), (3, 3, 128), (4, 2, 64), (6, 2, 128), (5, 1, 64),
                                      (7, 1, 128)])
def test_cache_heads_with_tails(dtype, group, hq, hkv, d):
    lens, tl = (77, 0, 300, 33), (5, 0, 40, 64)
    cake = context(hq, hkv, d, dtype, layers=3)
    check_cached(cake, cached(hq, hkv, d, dtype, lens, group, tail=(40, np.array(tl)), layers=3, layer=2), dtype)


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("group", [0, 32])
def test_cache_many_requests_and_one_long(dtype, group):
    """Work split over the device: far more heads than SMs, one of them much longer than the others; tails alone."""
    rng = np.random.default_rng(5)
    lens = [int(n) for n in rng.integers(0, 90, size=150)]
    lens[17] = 4000
    tl = rng.integers(-3, 30, size=150)
    cake = context(4, 2, 64, dtype, layers=2)
    check_cached(cake, cached(4, 2, 64, dtype, lens, group, tail=(20, tl)), dtype)
    check_cached(cake, cached(4, 2, 64, dtype, [0] * 5, group, tail=(20, tl[:5])), dtype)


@pytest.mark.parametrize("group", [0, 32])
def test_cache_results_do_not_depend_on_the_workspace_or_the_stream(group):
    x = cached(8, 2, 128, BF16, (700, 20, 1300), group, tail=(8, np.array([8, 0, 3])))
    cake = context(8, 2, 128, BF16, layers=2)
    out, lse = run_cached(cake, x)
    junk = torch.full((1 << 20,), float("nan"), device="cuda")       # freed: the next workspace may lie here
    del junk
    o2, l2 = run_cached(cake, x)
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    streams, got = [torch.cuda.Stream() for _ in range(4)], []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(5):
                got.append(run_cached(cake, x))
    torch.cuda.synchronize()
    assert all(torch.equal(o, out) and torch.equal(l, lse) for o, l in got)
    graph = torch.cuda.CUDAGraph()
    o3, l3 = torch.zeros_like(out), torch.zeros_like(lse)
    with torch.cuda.graph(graph):
        run_cached(cake, x, out=o3, lse=l3)
    x["q"].mul_(-1)
    graph.replay()
    o4, l4 = run_cached(cake, x)
    assert torch.equal(o3, o4) and torch.equal(l3, l4) and not torch.equal(o3, out)


def test_cache_refusals():
    cake = context(4, 2, 64, BF16, layers=2)
    x = cached(4, 2, 64, BF16, (40, 3), tail=(4, np.array([1, 2])))
    y = cached(4, 2, 64, BF16, (40, 3), group=32)
    run_cached(cake, x)
    run_cached(cake, y)
    for layer in (-1, 2):
        with pytest.raises(CakeError) as e:
            cake.attend_cache(layer, x["q"], x["k"], x["v"], x["off"])
        assert e.value.code == CAKE_ERR_ARG
        with pytest.raises(CakeError):
            cake.attend_int4(layer, y["q"], y["cache"])
    for bad in [dict(q=x["q"].float()), dict(q=x["q"][:, :3].contiguous()), dict(off=x["off"][:-1]), dict(off=x["off"].int()),
                dict(k=x["k"].float()), dict(k=x["k"].cpu())]:
        z = dict(x, **bad)
        with pytest.raises(ValueError):
            cake.attend_cache(1, z["q"], z["k"], z["v"], z["off"])
    for name in ("k_tail", "v_tail", "tail_len"):
        with pytest.raises(ValueError):
            cake.attend_cache(1, x["q"], x["k"], x["v"], x["off"], **dict(x["tail"], **{name: None}))
    for bad in [dict(k_codes=y["cache"]["k_codes"][:, :16].contiguous()), dict(v_scale=y["cache"]["v_scale"][:5]),
                dict(k_zero=y["cache"]["k_zero"][:1]), dict(kgroup_offsets=y["cache"]["kgroup_offsets"][:2])]:
        with pytest.raises(ValueError):
            cake.attend_int4(1, y["q"], dict(y["cache"], **bad))
    sixteen = torch.ones(y["cache"]["v_codes"].shape[0], 4, device="cuda")       # groups of 16 channels
    with pytest.raises(CakeError):
        cake.attend_int4(1, y["q"], dict(y["cache"], v_scale=sixteen, v_zero=sixteen))
    flat = torch.zeros(2 * 4 * 64 + 1, dtype=BF16, device="cuda")
    with pytest.raises(CakeError):
        cake.attend_cache(1, flat[1:].view(2, 4, 64), x["k"], x["v"], x["off"])
    lib, vp = cake.lib, (lambda t: t.data_ptr())
    ws = torch.empty(16, dtype=torch.uint8, device="cuda")
    need = lib.cake_attend_workspace_bytes(cake._h, 2)
    assert need > 0 and lib.cake_attend_workspace_bytes(cake._h, -1) == CAKE_ERR_ARG
    assert lib.cake_attend_cache(cake._h, 2, 1, vp(x["q"]), vp(x["k"]), vp(x["v"]), vp(x["off"]), None, None, None, 0,
                                 vp(torch.empty_like(x["q"])), None, vp(ws), 0, None) == binding.CAKE_ERR_CAPACITY
    out, lse = cake.attend_cache(0, x["q"][:0], x["k"], x["v"], x["off"][:1])
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)


# ------------------------------------------------------------------ together, as they are used
@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
def test_prefill_with_log_sum_exps_then_cached_attention(dtype):
    """attend_prompt -> score from its log-sum-exps -> cascade -> compaction in both forms -> attention of a new token."""
    d, hq, hkv, L, sw = 64, 8, 2, 3, 16
    lens = (400, 170)
    cu = [0, 400, 570]
    cake = context(hq, hkv, d, dtype, lens, window=sw, layers=L, budget=L * 60)
    layers = [prompt(hq, hkv, d, dtype, lens, seed=l) for l in range(L)]
    for l, (q, k, v) in enumerate(layers):
        lw = torch.empty(len(lens), hq, sw, device="cuda")
        cake.attend_prompt(q, k, v, lse_window=lw)
        qw = torch.stack([q[:, cu[r + 1] - sw:cu[r + 1]] for r in range(len(lens))]).contiguous()
        cake.score_layer(l, qw, k, lse=lw)
        cake.allocate(l)
        cake.evict(l)
    P = cake.get_preferences()[2].cpu().numpy()
    for r in range(len(lens)):
        for l, (q, k, v) in enumerate(layers):
            qn, kn = f64(q)[:, cu[r + 1] - sw:cu[r + 1]], f64(k)[:, cu[r]:cu[r + 1]]
            want = O.score_layer(qn, kn, gamma=200.0, pool_kernel=1, tau1=1.0, tau2=1.0)["P"]
            assert abs(P[r, l] - want) <= 1e-3 * want
    ks, vs = [x[1] for x in layers], [x[2] for x in layers]
    k_out, v_out, off, _ = cake.compact(ks, vs)
    q4 = cake.compact_int4(ks, vs, group=32)
    offn, koff = off.cpu().numpy(), q4["kgroup_offsets"].cpu().numpy()
    q_new = torch.randn(len(lens), hq, d, device="cuda").to(dtype)
    for l in range(L):
        for int4 in (False, True):
            out, lse = cake.attend_int4(l, q_new, q4) if int4 else cake.attend_cache(l, q_new, k_out, v_out, off)
            for r in range(len(lens)):
                a, b = offn[r * L + l], offn[r * L + l + 1]
                n = (b - a) // hkv
                for g in range(hkv):
                    rows = slice(a + g * n, a + (g + 1) * n)
                    k, v = f64(k_out[rows]), f64(v_out[rows])
                    if int4:
                        gn = -(-n // 32)
                        ga = koff[r * L + l] + g * gn
                        code = lambda name: O.unpack_nibbles(q4[name][rows].cpu().numpy())
                        k = O.dequantize_keys(code("k_codes"), q4["k_scale"][ga:ga + gn].cpu().numpy(),
                                              q4["k_zero"][ga:ga + gn].cpu().numpy(), 32)
                        v = O.dequantize_values(code("v_codes"), q4["v_scale"][rows].cpu().numpy(),
                                                q4["v_zero"][rows].cpu().numpy(), 32)
                    heads = slice(g * 4, g * 4 + 4)
                    want = O.attend(f64(q_new)[r, heads], k, v)
                    dw = weight_error(f64(q_new)[r, heads], 2 * np.abs(k), d) + 2.0 ** -16 * int4 * 8
                    check_out(f64(out)[r, heads], f64(lse)[r, heads], (want[0], want[1], np.maximum(want[2], np.abs(v).max())),
                              dw, n, dtype)


def test_eviction_by_accumulated_attention():
    """The accumulated weights as indicators: what is kept are each head's heaviest tokens and the window."""
    d, hq, hkv, L, sw = 128, 8, 2, 2, 8
    lens = (300, 500)
    cu = [0, 300, 800]
    cake = context(hq, hkv, d, BF16, lens, window=sw, layers=L, budget=L * 64, alloc_mode=1)
    cake.set_preferences(torch.ones(len(lens), L, dtype=torch.float64, device="cuda"))
    received, layers = [], [prompt(hq, hkv, d, BF16, lens, seed=10 + l) for l in range(L)]
    for l, (q, k, v) in enumerate(layers):
        received.append(cake.accumulate_attention(q, k, cake.attend_prompt(q, k, v)[1]))
        cake.set_indicators(l, received[-1])
        cake.allocate(l)
        cake.evict(l)
    budgets = cake.get_budgets().cpu().numpy()
    for r in range(len(lens)):
        for l in range(L):
            n = lens[r] - sw
            got = cake.get_positions(r, l, int(budgets[r, l])).cpu().numpy()
            for g in range(hkv):
                ind = f64(received[l])[g, cu[r]:cu[r] + n]
                keep = O.topk_keep(ind, int(budgets[r, l]) - sw)
                assert np.array_equal(got[g], np.concatenate([keep, np.arange(n, lens[r])]))
    assert cake.status() == 0


def test_attention_output_of_a_decode_step():
    """After a step of decode-time eviction the block's slots hold the rows that the new token has attended."""
    d, hq, hkv, L, sw = 128, 8, 2, 2, 8
    lens = (200, 90)
    w = synth.scaled(synth.workload(3), n_layers=L, n_q_heads=hq, n_kv_heads=hkv, seq_lens=lens, total_budget=L * 48, window=sw)
    qs, ks, vs = harness.device_inputs(w)
    cake = harness.cake_for(w)
    cake.run(qs, ks, vs, w.cu_seqlens)
    kc, vc, off = cake.decode_begin(ks, vs)
    g = torch.Generator().manual_seed(1)
    for _ in range(3):
        for l in range(L):
            q, k, v = (torch.randn(2, h, d, generator=g).to(BF16).cuda() for h in (hq, hkv, hkv))
            cake.decode_step(l, q, k, v, kc, vc)
            out, lse = cake.attend_cache(l, q, kc, vc, off)
            o = off.cpu().numpy()
            for r in range(2):
                a, b = o[r * L + l], o[r * L + l + 1]
                n = (b - a) // hkv
                for h in range(hkv):
                    rows = slice(a + h * n, a + (h + 1) * n)
                    assert (kc[rows] == k[r, h]).all(1).any()         # the new token's row is among them
                    want = O.attend(f64(q)[r, h * 4:h * 4 + 4], f64(kc[rows]), f64(vc[rows]))
                    dw = weight_error(f64(q)[r, h * 4:h * 4 + 4], f64(kc[rows]), d)
                    check_out(f64(out)[r, h * 4:h * 4 + 4], f64(lse)[r, h * 4:h * 4 + 4], want, dw, n, BF16)


# ------------------------------------------------------------------ large
@pytest.mark.parametrize("dtype,n", [(BF16, 20011), (FP32, 9001)], ids=["bf16", "fp32"])
def test_long_prompt_rows(dtype, n):
    """Rows of a long prompt, at the tiles' borders and between, and the columns' sums from the device's own rows."""
    cake = context(4, 2, 128, dtype, (n,))
    q, k, v = prompt(4, 2, 128, dtype, (n,))
    out, lse = cake.attend_prompt(q, k, v)
    kn, vn = f64(k), f64(v)
    rows = [0, 127, 128, 255, 256, 8191, 8192, n - 130, n - 2, n - 1] + list(np.random.default_rng(1).integers(0, n, 20))
    for h in range(4):
        for i in rows:
            want = O.attend(f64(q[h, i:i + 1]), kn[h // 2, :i + 1], vn[h // 2, :i + 1])
            dw = weight_error(f64(q[h, i:i + 1]), kn[h // 2, :i + 1], 128)
            check_out(f64(out[h, i:i + 1]), f64(lse[h, i:i + 1]), want, dw, i + 1, dtype)
    got = f64(cake.accumulate_attention(q, k, lse))
    ln, qn = f64(lse), f64(q)
    for j in (0, 5, 127, 128, 4099, n - 64, n - 1):
        for g in range(2):
            s = (qn[2 * g:2 * g + 2, j:] @ kn[g, j]) / np.sqrt(128.0)
            ref = np.exp(s - ln[2 * g:2 * g + 2, j:]).sum() / 2
            dw = weight_error(qn[2 * g:2 * g + 2], kn[g, j:j + 1], 128)
            assert abs(got[g, j] - ref) <= (2 * dw + 4 * U * np.abs(ln).max() + 2 * n * U) * ref


@pytest.mark.parametrize("group", [0, 32])
def test_cache_offsets_beyond_32_bits(group):
    """The block lies beyond 2^31 elements (bytes of codes) of its buffers."""
    d, n, first = 128, 700, 17_000_000 if group == 0 else 34_000_000
    rows = first + 2 * n
    cake = context(8, 2, d, BF16, layers=2)
    x = cached(8, 2, d, BF16, (n,), group, layers=1, layer=0)
    x["layer"] = 1
    far = torch.tensor([0, first, rows], dtype=torch.int64, device="cuda")
    if group == 0:
        big = {m: torch.empty(rows, d, dtype=BF16, device="cuda") for m in "kv"}
        for m in "kv":
            big[m][first:] = x[m][:2 * n]
        got = cake.attend_cache(1, x["q"], big["k"], big["v"], far)
        want = context(8, 2, d, BF16).attend_cache(0, x["q"], x["k"], x["v"], x["off"])
    else:
        c = x["cache"]
        groups = 2 * -(-n // group)
        big = {m: torch.empty(rows, *t.shape[1:], dtype=t.dtype, device="cuda") for m, t in c.items() if m in ("k_codes", "v_codes", "v_scale", "v_zero")}
        for m in big:
            big[m][first:] = c[m][:2 * n]
        start = first // group
        for m in ("k_scale", "k_zero"):
            big[m] = torch.empty(start + groups, d, device="cuda")
            big[m][start:] = c[m][:groups]
        big.update(row_offsets=far, kgroup_offsets=torch.tensor([0, start, start + groups], dtype=torch.int64, device="cuda"))
        got = cake.attend_int4(1, x["q"], big)
        want = context(8, 2, d, BF16).attend_int4(0, x["q"], c)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_prompt_offsets_beyond_32_bits(layout):
    """The last requests of a batch whose queries and outputs have more than 2^31 elements."""
    hq, hkv, d, many, each = 16, 2, 128, 1200, 900
    lens = (each,) * many
    T = sum(lens)
    cake = context(hq, hkv, d, BF16, lens)
    q = torch.zeros((hq, T, d) if layout == "heads" else (T, hq, d), dtype=BF16, device="cuda")
    q = q if layout == "heads" else q.transpose(0, 1)
    k, v = torch.zeros(hkv, T, d, dtype=BF16, device="cuda"), torch.zeros(hkv, T, d, dtype=BF16, device="cuda")
    qs, ks, vs = prompt(hq, hkv, d, BF16, (each, each))
    q[:, T - 2 * each:], k[:, T - 2 * each:], v[:, T - 2 * each:] = qs, ks, vs
    out, lse = cake.attend_prompt(q, k, v)
    got = cake.accumulate_attention(q, k, lse)
    small = context(hq, hkv, d, BF16, (each, each))
    want, want_lse = small.attend_prompt(qs, ks, vs)
    assert q.numel() > 2 ** 31
    assert torch.equal(out[:, T - 2 * each:], want) and torch.equal(lse[:, T - 2 * each:], want_lse)
    one = got[:, T - 2 * each:]
    ref = small.accumulate_attention(qs, ks, want_lse)
    assert (one - ref).abs().max() <= 1e-5 * ref.abs().max()       # (few keys: their heads are split over CTAs)
    cake.destroy()


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,d", [(5, 1, 64), (7, 1, 128), (10, 2, 128)])
def test_prompt_groups_of_odd_size(hq, hkv, d, dtype):
    lens = (150, 290)
    cake = context(hq, hkv, d, dtype, lens, window=4)
    check_prompt(cake, *prompt(hq, hkv, d, dtype, lens, seed=hq), lens, dtype, window=4)


@pytest.mark.parametrize("group", [0, 32])
def test_cache_thousands_of_requests(group):
    """More requests than a warp reads at once, most of them short or empty."""
    rng = np.random.default_rng(11)
    lens = [int(n) for n in rng.integers(0, 4, size=3000)]
    lens[2999] = 500
    cake = context(2, 1, 64, BF16, layers=2)
    check_cached(cake, cached(2, 1, 64, BF16, lens, group), BF16)


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
def test_cache_logits_of_minus_infinity(dtype):
    """Keys whose logit is -inf weigh nothing, also where a whole unit of rows has no other; only a request of such keys alone has
    no answer."""
    lens, d = (200, 33, 5), 64
    x = cached(4, 2, d, dtype, lens, seed=9)
    x["q"][:, :, 0] = 1
    bad = [np.r_[0:64, 100:140, 199], np.r_[32], np.r_[0:5]]
    for r, n in enumerate(lens):
        for g in range(2):
            x["k"][int(x["offn"][r * 2 + 1]) + g * n + torch.from_numpy(bad[r]).cuda(), 0] = float("-inf")
    out, lse = run_cached(context(4, 2, d, dtype, layers=2), x)
    assert torch.isnan(out[2]).all() and (lse[2] == float("-inf")).all()
    on, ln, qn = f64(out), f64(lse), f64(x["q"])
    for r, n in enumerate(lens[:2]):
        for g in range(2):
            keep = int(x["offn"][r * 2 + 1]) + g * n + np.setdiff1d(np.arange(n), bad[r])
            k, v, heads = x["kn"][keep], x["vn"][keep], slice(2 * g, 2 * g + 2)
            check_out(on[r, heads], ln[r, heads], O.attend(qn[r, heads], k, v), weight_error(qn[r, heads], k, d), n, dtype)


def test_prompt_logits_of_minus_infinity():
    n, bad, d = 700, 270, 64
    cake = context(2, 1, d, BF16, (n,))
    q, k, v = prompt(2, 1, d, BF16, (n,), seed=4)
    q[:, :, 0] = 1
    k[:, :bad, 0] = float("-inf")
    out, lse = cake.attend_prompt(q, k, v)
    assert torch.isnan(out[:, :bad]).all() and (lse[:, :bad] == float("-inf")).all()
    qn, kn, vn = f64(q[:, bad:]), f64(k[:, bad:]), f64(v[:, bad:])
    check_out(f64(out[:, bad:]), f64(lse[:, bad:]), O.prompt_attention(qn, kn, vn), weight_error(qn, kn, d), n, BF16)


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("group", [0, 32])
def test_cache_of_tails_alone(dtype, group):
    """No packed row at all: the cache's tensors have no memory."""
    cake = context(4, 2, 64, dtype, layers=1)
    x = cached(4, 2, 64, dtype, (0, 0), group=group, tail=(7, np.array([7, 3])), layers=1, layer=0)
    if group:
        x["cache"] = {n: t if n.endswith("offsets") else t[:0] for n, t in x["cache"].items()}
        x["cache"] = {n: t if n.endswith("offsets") else torch.empty_like(t) for n, t in x["cache"].items()}
    else:
        x["k"], x["v"] = (torch.empty((0, 64), dtype=dtype, device="cuda") for _ in range(2))
    check_cached(cake, x, dtype)


@pytest.mark.parametrize("group", [0, 32])
def test_calls_among_copies_and_other_streams_in_a_graph(group):
    """A captured step whose kernels follow copies, a fill and a join of two streams, several times behind one another: the same
    as one by one, whatever of it may start early."""
    lens = (700, 40)
    cake = context(8, 2, 128, BF16, lens, layers=2)
    q, k, v = prompt(8, 2, 128, BF16, lens, seed=2)
    x = cached(8, 2, 128, BF16, (900, 130, 33), group=group, tail=(9, np.array([9, 0, 4])), seed=8)
    queries = x["q"].clone()

    def step(side):
        main = torch.cuda.current_stream()
        got = []
        lse = torch.zeros(8, sum(lens), device="cuda")
        x["q"].copy_(queries)
        got += run_cached(cake, x)
        side.wait_stream(main)
        with torch.cuda.stream(side):
            first = cake.attend_prompt(q, k, v, lse=lse)
            received = cake.accumulate_attention(q, k, lse)
        x["q"].mul_(0.5)
        got += run_cached(cake, x)
        main.wait_stream(side)
        got += run_cached(cake, x)
        got += [first[0], lse, received, cake.accumulate_attention(q, k, lse)]
        return got

    side = torch.cuda.Stream()
    want = [t.clone() for t in step(side)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(side)
    for _ in range(3):
        for t in got:
            t.fill_(7)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("group", [0, 32])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 1, 64), (16, 16, 64)])
def test_cache_short_ragged_requests_repeat_bit_for_bit(hq, hkv, d, group):
    """Many pairs end inside a CTA, of one unit or of a few more than it has warps: whichever warp puts results together, and when."""
    rng = np.random.default_rng(hq + d + group)
    lens = tuple(int(n) for n in rng.choice([0, 1, 20, 33, 64, 65, 130, 260, 300, 390, 600], size=250))
    cake = context(hq, hkv, d, BF16, layers=1)
    x = cached(hq, hkv, d, BF16, lens, group=group, layers=1, layer=0, tail=(20, rng.integers(0, 21, size=250)))
    out, lse = check_cached(cake, x, BF16)
    for _ in range(40):
        again, lse2 = run_cached(cake, x)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    assert cake.status() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_calls_on_two_streams_at_once(d):
    """Prompts of one context beside prompts and caches of another, on streams of their own: the same as one by one."""
    lens, group = (1500, 260), 32
    work = []
    for dtype in (BF16, FP32):
        x = cached(8, 2, d, dtype, (900, 130, 33), group=group, tail=(9, np.array([9, 0, 4])), seed=8)
        work.append((context(8, 2, d, dtype, lens, layers=2), prompt(8, 2, d, dtype, lens, seed=d), x))

    def step(cake, qkv, x):
        out, lse = cake.attend_prompt(*qkv)
        return out, lse, cake.accumulate_attention(qkv[0], qkv[1], lse), *run_cached(cake, x)

    want = [step(*w) for w in work]
    streams = [torch.cuda.Stream() for _ in work]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for s, w in zip(streams, work):
            with torch.cuda.stream(s):
                got.append(step(*w))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[i % 2]))
    assert all(cake.status() == 0 for cake, *_ in work)
