"""Timed cases of the attention operators that surround the eviction path.

A case is a dict of plain values; `kind` says which operator it exercises:

  prompt      causal attention over whole prompts of a packed batch, grouped heads: the output and every row's
              log-sum-exp, which the window scoring takes in place of its own first pass.
  accumulate  the attention weight that every key has received from all queries of its prompt (from those
              log-sum-exps), averaged over the query heads of its KV head: the indicator of an eviction by
              accumulated attention.
  cache       attention of one new token per request over the packed cache of retained rows (and over the rows of
              tokens generated since, where there are any).
  int4        the same over the cache held in 4 bits: keys quantised per channel, values per token.

`own` says whose code `run` calls: False computes the operators from elementary torch operations in 32 bits, True calls
the library.
"""
import math
import random

import torch

own = False


# ------------------------------------------------------------------ the cases
def _prompt(kind, **kw):
    # layout "tokens": the queries lie as a projection leaves them, [token][head][channel]; "heads": [head][token][channel]
    c = dict(kind=kind, q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", layout="tokens", requests=1, shortest=4096,
             longest=4096)
    c.update(kw)
    return c


def _cached(kind, **kw):
    # lengths are retained rows per KV head; `tail` is the room for generated tokens per request (0: none)
    c = dict(kind=kind, q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", requests=1, shortest=2048, longest=2048,
             tail=0)
    if kind == "int4":
        c["group"] = 32
    c.update(kw)
    return c


def listed():
    return [
        # a long-document prompt of a grouped-query model: one layer's attention
        _prompt("prompt", name="prompt-gqa-32k", shortest=32768, longest=32768),
        # multi-head attention at 4K
        _prompt("prompt", name="prompt-mha-4k", kv_heads=32),
        # a server's batch of short prompts of odd lengths
        _prompt("prompt", name="prompt-ragged", requests=8, shortest=257, longest=7919),
        # the smallest configuration: 512 tokens in fp32, where launches and latency count
        _prompt("prompt", name="prompt-tiny-fp32", q_heads=4, kv_heads=4, head_dim=64, dtype="fp32", layout="heads",
                shortest=512, longest=512),
        # accumulated attention of a 16K prompt
        _prompt("accumulate", name="accumulate-gqa-16k", shortest=16384, longest=16384),
        # the same for a ragged batch of short prompts
        _prompt("accumulate", name="accumulate-ragged", requests=4, shortest=1501, longest=7919),
        # fp32 inputs: research use and the numerics baseline
        _prompt("accumulate", name="accumulate-fp32-6k", q_heads=16, kv_heads=4, dtype="fp32", layout="heads",
                shortest=6001, longest=6001),
        # a token of one user's answer over the rows that a budget of 2048 left
        _cached("cache", name="cache-one-2k"),
        # a server's batch: ragged budgets, some tokens generated already
        _cached("cache", name="cache-batch32", requests=32, shortest=1000, longest=6000, tail=64),
        # the 128K prompt's budget in 4 bits, one user
        _cached("int4", name="int4-one-4k", shortest=4096, longest=4096),
        # the same for a server's batch
        _cached("int4", name="int4-batch32", requests=32, shortest=1000, longest=8000, tail=64),
        # small heads, multi-head attention, coarser groups, odd lengths
        _cached("int4", name="int4-mha-d64", q_heads=16, kv_heads=16, head_dim=64, requests=8, shortest=777, longest=4099,
                group=64),
    ]


def _log_int(rng, lo, hi):
    """An integer spread evenly over the logarithm of lo..hi."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# (query heads, KV heads, head_dim) in use: grouped-query and multi-head models
_HEADS_BF16 = [(32, 8, 128), (32, 32, 128), (16, 2, 128), (16, 8, 128), (16, 16, 64), (8, 8, 128)]
_HEADS_FP32 = [(4, 4, 64), (16, 4, 128), (8, 8, 64), (8, 2, 128)]


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "accumulate", "cache", "int4", "int4"])
    fp32 = rng.random() < 0.25
    q_heads, kv_heads, head_dim = rng.choice(_HEADS_FP32 if fp32 else _HEADS_BF16)
    requests = rng.choice([1, 1, 2, 4, 8] if kind in ("prompt", "accumulate") else [1, 1, 2, 8, 32])
    shape = dict(q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, dtype="fp32" if fp32 else "bf16", requests=requests)
    if kind in ("prompt", "accumulate"):
        most = 4096 if fp32 else 16384
        longest = _log_int(rng, 64, most // requests if requests > 2 else most)
        return _prompt(kind, shortest=longest if requests == 1 else max(33, longest // rng.choice([1, 2, 8])),
                       longest=longest, layout=rng.choice(["tokens", "heads"]), **shape)
    longest = _log_int(rng, 16, 65536 // requests)
    c = _cached(kind, shortest=longest if requests == 1 else max(1, longest // rng.choice([1, 2, 8])), longest=longest,
                tail=rng.choice([0, 16, 256]), **shape)
    if kind == "int4":
        c["group"] = rng.choice([g for g in (32, 64, 128) if g <= head_dim])
    return c


# ------------------------------------------------------------------ inputs
_LAYERS, _LAYER = 2, 1             # the caches hold two layers, of which the second is read


def _lengths(case):
    """Prompt lengths, or retained rows per head and request: a property of the case, not of the seed."""
    lo, hi = case["shortest"], case["longest"]
    if case["requests"] == 1:
        return [hi]
    r = random.Random(lo * 1000003 + hi * 101 + case["requests"])
    return [hi] + [r.randint(lo, hi) for _ in range(case["requests"] - 1)]


def _tails(case):
    r = random.Random(case["longest"] * 31 + case["tail"])
    return [r.randint(0, case["tail"]) for _ in range(case["requests"])]


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _temperature(seed):
    """Standard deviation of the logits: layers range from nearly uniform to sharp attention."""
    return math.exp(random.Random(seed).uniform(math.log(0.5), math.log(4.0)))


def _keys(case, gen, rows, direction, boost):
    """Keys of one layer [KV head][row][channel]; `boost` [row] moves a row along its head's mean query."""
    k = _randn(gen, case["kv_heads"], rows, case["head_dim"])
    return k + boost[None, :, None] * (2.0 / math.sqrt(case["head_dim"])) * direction[:, None, :]


def _prompt_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens = _lengths(case)
    cu, t = _cu(lens), _temperature(seed)
    hq, hkv, d, total = case["q_heads"], case["kv_heads"], case["head_dim"], sum(lens)
    direction = _randn(gen, hkv, d)
    boost = (torch.rand(total, generator=gen, device="cuda") < 0.01).float() * 2.0      # heavy hitters
    for r, n in enumerate(lens):
        boost[cu[r]:cu[r] + min(4, n)] = 3.0                                            # sink tokens
    k = _keys(case, gen, total, direction, boost).to(_dtype(case))
    v = _randn(gen, hkv, total, d).to(_dtype(case))
    mean = 0.5 * direction.repeat_interleave(hq // hkv, 0)
    if case["layout"] == "tokens":
        q = (t * (_randn(gen, total, hq, d) + mean)).to(_dtype(case)).transpose(0, 1)
    else:
        q = (t * (_randn(gen, hq, total, d) + mean[:, None, :])).to(_dtype(case))
    return dict(q=q, k=k, v=v, cu=cu)


def _quantize(x, dim):
    """4-bit codes of the groups along `dim`, their scale and zero."""
    zero = x.amin(dim, keepdim=True)
    span = x.amax(dim, keepdim=True) - zero
    scale = torch.where(span > 0, span / 15.0, torch.ones_like(span))
    code = torch.round((x - zero) / scale).clamp_(0, 15).to(torch.uint8)
    return code, scale, zero


def _nibbles(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _cache_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens, tails = _lengths(case), _tails(case)
    n_req, hq, hkv, d, dt = case["requests"], case["q_heads"], case["kv_heads"], case["head_dim"], _dtype(case)
    t, direction = _temperature(seed), _randn(gen, hkv, d)
    blocks = [n // 2 + 1 if l != _LAYER else n for n in lens for l in range(_LAYERS)]   # rows per head of (request, layer)
    rows = _cu([hkv * n for n in blocks])
    total = rows[-1]
    k = torch.empty(total, d, device="cuda")
    for i, n in enumerate(blocks):
        boost = (torch.rand(n, generator=gen, device="cuda") < 0.1).float()             # retained rows: many heavy hitters
        boost[:min(4, n)] = 3.0
        k[rows[i]:rows[i + 1]] = _keys(case, gen, n, direction, boost).reshape(-1, d)
    v = _randn(gen, total, d)
    x = dict(n_req=n_req, rows=rows, row_offsets=torch.tensor(rows, dtype=torch.int64, device="cuda"),
             q=(t * (_randn(gen, n_req, hq, d) + 0.5 * direction.repeat_interleave(hq // hkv, 0))).to(dt),
             k_tail=None, v_tail=None, tail_len=None)
    if case["tail"]:
        x["k_tail"] = _randn(gen, n_req, hkv, case["tail"], d).to(dt)
        x["v_tail"] = _randn(gen, n_req, hkv, case["tail"], d).to(dt)
        x["tail_len"] = torch.tensor(tails, dtype=torch.int32, device="cuda")
    if case["kind"] == "cache":
        return dict(x, k=k.to(dt), v=v.to(dt))
    g = case["group"]
    k, v = k.to(dt).float(), v.to(dt).float()
    vc, vs, vz = _quantize(v.view(total, d // g, g), 2)
    groups = _cu([hkv * -(-n // g) for n in blocks])
    kc = torch.empty(total, d, dtype=torch.uint8, device="cuda")
    ks, kz = torch.empty(groups[-1], d, device="cuda"), torch.empty(groups[-1], d, device="cuda")
    for i, n in enumerate(blocks):
        per = -(-n // g)
        blk = k[rows[i]:rows[i + 1]].view(hkv, n, d)
        # a head's last group may be shorter: a repeated last row changes neither its range nor its codes
        pad = torch.cat([blk, blk[:, -1:].expand(hkv, per * g - n, d)], 1).reshape(hkv * per, g, d)
        code, scale, zero = _quantize(pad, 1)
        kc[rows[i]:rows[i + 1]] = code.view(hkv, per * g, d)[:, :n].reshape(-1, d)
        ks[groups[i]:groups[i + 1]], kz[groups[i]:groups[i + 1]] = scale.squeeze(1), zero.squeeze(1)
    cache = dict(k_codes=_nibbles(kc).contiguous(), k_scale=ks, k_zero=kz,
                 v_codes=_nibbles(vc.view(total, d)).contiguous(), v_scale=vs.view(total, -1), v_zero=vz.view(total, -1),
                 row_offsets=x["row_offsets"],
                 kgroup_offsets=torch.tensor(groups, dtype=torch.int64, device="cuda"))
    return dict(x, cache=cache, groups=groups, group=g)


def _inputs(case, seed):
    if case["kind"] in ("cache", "int4"):
        return _cache_inputs(case, seed)
    x = _prompt_inputs(case, seed)
    if case["kind"] == "accumulate":
        x["lse"] = _row_lse(x)                       # as the attention over the prompt leaves them
    return x


def _context(case, x):
    """The library's context of a user's program, with the batch begun where there is one."""
    from paper_2503_12491_b200 import Cake
    cached = case["kind"] in ("cache", "int4")
    window = min(32, min(_lengths(case)), 128 * case["kv_heads"] // case["q_heads"])
    cake = Cake(n_layers=_LAYERS if cached else 1, n_q_heads=case["q_heads"], n_kv_heads=case["kv_heads"],
                head_dim=case["head_dim"], window=window, pool_kernel=1, gamma=200.0, total_budget=4096,
                max_requests=case["requests"], max_total_tokens=256 * case["requests"] if cached else x["cu"][-1],
                dtype=_dtype(case))
    if not cached:
        cake.begin(x["cu"])
    return cake


def prepare(case, seed):
    x = dict(_inputs(case, seed), kind=case["kind"], heads=(case["q_heads"], case["kv_heads"]))
    if own:
        x["cake"] = _context(case, x)
    return x


# ------------------------------------------------------------------ one pass
_CHUNK = 256 << 20                  # logits held at once by the plain form


def _chunks(x):
    """(request's first and last token, query rows of a chunk), the latter relative to the request."""
    hq = x["q"].shape[0]
    for a, b in zip(x["cu"], x["cu"][1:]):
        step = max(1, min(b - a, _CHUNK // (hq * (b - a))))
        for lo in range(0, b - a, step):
            yield a, b, lo, min(lo + step, b - a)


def _logits(x, a, lo, hi):
    """Causal logits of query rows lo..hi of the request that starts at token a, over its keys 0..hi:
    [KV head][query head of its group * row][key], -inf where a key lies behind the row."""
    q, k = x["q"][:, a + lo:a + hi].float(), x["k"][:, a:a + hi].float()
    hq, n, d = q.shape
    s = torch.bmm(q.reshape(k.shape[0], -1, d), k.transpose(1, 2)).mul_(1.0 / math.sqrt(d)).view(hq, n, hi)
    behind = torch.arange(hi, device=q.device)[None, :] > torch.arange(lo, hi, device=q.device)[:, None]
    return s.masked_fill_(behind, -math.inf).view(k.shape[0], -1, hi)


def _softmax_parts(s):
    top = s.amax(-1, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    return p, total, (top + total.log()).squeeze(-1)


def _row_lse(x):
    lse = torch.empty(x["q"].shape[:2], device="cuda")
    for a, _, lo, hi in _chunks(x):
        lse[:, a + lo:a + hi] = _softmax_parts(_logits(x, a, lo, hi))[2].view(-1, hi - lo)
    return lse


def _plain_prompt(x):
    q = x["q"]
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    for a, _, lo, hi in _chunks(x):
        p, total, row = _softmax_parts(_logits(x, a, lo, hi))
        o = torch.bmm(p, x["v"][:, a:a + hi].float()) / total
        out[:, a + lo:a + hi] = o.view(q.shape[0], hi - lo, -1).to(q.dtype)
        lse[:, a + lo:a + hi] = row.view(-1, hi - lo)
    return out, lse


def _plain_accumulate(x):
    hkv, total = x["k"].shape[:2]
    got = torch.zeros(hkv, total, dtype=torch.float64, device="cuda")
    for a, _, lo, hi in _chunks(x):
        row = x["lse"][:, a + lo:a + hi].reshape(hkv, -1, 1)
        got[:, a:a + hi] += _logits(x, a, lo, hi).sub_(row).exp_().sum(1)
    return (got * (hkv / x["q"].shape[0])).float()


def _codes(packed):
    return torch.stack((packed & 15, packed >> 4), -1).flatten(-2).float()


def _cached_rows(x, r):
    """K and V of a request's retained rows in 32 bits, [KV head][row][channel]."""
    i, hkv = r * _LAYERS + _LAYER, x["heads"][1]
    a, b = x["rows"][i], x["rows"][i + 1]
    n = (b - a) // hkv
    if x["kind"] == "cache":
        return x["k"][a:b].view(hkv, n, -1).float(), x["v"][a:b].view(hkv, n, -1).float()
    c, g = x["cache"], x["group"]
    d = c["k_codes"].shape[1] * 2
    ga, gb = x["groups"][i], x["groups"][i + 1]
    of_row = torch.arange(n, device="cuda") // g
    k = c["k_zero"][ga:gb].view(hkv, -1, d)[:, of_row] + \
        _codes(c["k_codes"][a:b]).view(hkv, n, d) * c["k_scale"][ga:gb].view(hkv, -1, d)[:, of_row]
    v = c["v_zero"][a:b, :, None] + _codes(c["v_codes"][a:b]).view(b - a, -1, g) * c["v_scale"][a:b, :, None]
    return k, v.reshape(hkv, n, d)


def _plain_cached(x):
    q = x["q"]
    n_req, hq, d = q.shape
    out, lse = torch.empty_like(q), torch.empty(n_req, hq, device="cuda")
    for r in range(n_req):
        k, v = _cached_rows(x, r)
        live = None
        if x["k_tail"] is not None:
            room = x["k_tail"].shape[2]
            live = torch.arange(k.shape[1] + room, device="cuda") < k.shape[1] + x["tail_len"][r]
            k = torch.cat([k, x["k_tail"][r].float()], 1)
            v = torch.cat([v, x["v_tail"][r].float()], 1)
        s = torch.bmm(q[r].float().view(k.shape[0], -1, d), k.transpose(1, 2)).mul_(1.0 / math.sqrt(d))
        if live is not None:
            s = s.masked_fill_(~live, -math.inf)
        p, total, row = _softmax_parts(s)
        out[r] = (torch.bmm(p, v) / total).view(hq, d).to(q.dtype)
        lse[r] = row.view(hq)
    return out, lse


def run(x):
    kind = x["kind"]
    if not own:
        return (_plain_prompt if kind == "prompt" else _plain_accumulate if kind == "accumulate" else _plain_cached)(x)
    cake = x["cake"]
    if kind == "prompt":
        return cake.attend_prompt(x["q"], x["k"], x["v"])
    if kind == "accumulate":
        return cake.accumulate_attention(x["q"], x["k"], x["lse"])
    tail = dict(k_tail=x["k_tail"], v_tail=x["v_tail"], tail_len=x["tail_len"])
    if kind == "cache":
        return cake.attend_cache(_LAYER, x["q"], x["k"], x["v"], x["row_offsets"], **tail)
    return cake.attend_int4(_LAYER, x["q"], x["cache"], **tail)


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    x = _inputs(case, seed)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] in ("cache", "int4"):
        return _exact_cached(case, x, hq // hkv)
    q, k, v = x["q"], x["k"], x["v"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    received = torch.zeros(k.shape[:2], dtype=torch.float64, device="cuda")
    for a, b in zip(x["cu"], x["cu"][1:]):
        for h in range(hq):
            g = h // (hq // hkv)
            kk, vv = k[g, a:b].double(), v[g, a:b].double()
            for lo in range(a, b, 2048):
                hi = min(lo + 2048, b)
                seen = torch.ones(hi - lo, hi - a, dtype=torch.bool, device="cuda").tril(lo - a)
                s = torch.where(seen, q[h, lo:hi].double() @ kk[:hi - a].T / math.sqrt(d), -math.inf)
                if case["kind"] == "prompt":
                    lse[h, lo:hi] = torch.logsumexp(s, 1)
                    out[h, lo:hi] = torch.exp(s - lse[h, lo:hi, None]) @ vv[:hi - a]
                else:
                    received[g, a:hi] += torch.exp(s - x["lse"][h, lo:hi, None].double()).sum(0) / (hq // hkv)
    return (out, lse) if case["kind"] == "prompt" else received


def _exact_cached(case, x, group):
    q = x["q"].double()
    n_req, hq, d = q.shape
    out = torch.zeros(n_req, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(n_req, hq, dtype=torch.float64, device="cuda")
    for r, tail in enumerate(_tails(case)):
        for g in range(case["kv_heads"]):
            block = r * _LAYERS + _LAYER
            n = (x["rows"][block + 1] - x["rows"][block]) // case["kv_heads"]
            at = x["rows"][block] + g * n
            if case["kind"] == "cache":
                k, v = x["k"][at:at + n].double(), x["v"][at:at + n].double()
            else:
                c, size = x["cache"], x["group"]
                first = x["groups"][block] + g * -(-n // size)
                k, v = (torch.zeros(n, d, dtype=torch.float64, device="cuda") for _ in range(2))
                for codes, into in ((c["k_codes"], k), (c["v_codes"], v)):
                    into[:, 0::2] = (codes[at:at + n] % 16).double()
                    into[:, 1::2] = (codes[at:at + n] // 16).double()
                for part in range(-(-n // size)):
                    rows = slice(part * size, min(n, part * size + size))
                    k[rows] = k[rows] * c["k_scale"][first + part].double() + c["k_zero"][first + part].double()
                for part in range(d // size):
                    cols = slice(part * size, part * size + size)
                    v[:, cols] = v[:, cols] * c["v_scale"][at:at + n, part, None].double() + \
                        c["v_zero"][at:at + n, part, None].double()
            if tail:
                k = torch.cat([k, x["k_tail"][r, g, :tail].double()])
                v = torch.cat([v, x["v_tail"][r, g, :tail].double()])
            heads = slice(g * group, g * group + group)
            s = q[r, heads] @ k.T / math.sqrt(d)
            lse[r, heads] = torch.logsumexp(s, 1)
            out[r, heads] = torch.exp(s - lse[r, heads, None]) @ v
    return out, lse


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    es = 4 if case["dtype"] == "fp32" else 2
    hq, hkv, d, lens = case["q_heads"], case["kv_heads"], case["head_dim"], _lengths(case)
    total = sum(lens)
    if case["kind"] in ("prompt", "accumulate"):
        pairs = hq * sum(n * (n + 1) // 2 for n in lens)
        if case["kind"] == "prompt":                 # q, k, v in; out and the log-sum-exps out
            return {"bytes": total * d * es * 2 * (hq + hkv) + 4 * hq * total, "flops": 4 * d * pairs}
        return {"bytes": total * d * es * (hq + hkv) + 4 * (hq + hkv) * total, "flops": 2 * d * pairs}
    tails = sum(_tails(case)) if case["tail"] else 0
    small = len(lens) * hq * (2 * d * es + 4) + tails * hkv * 2 * d * es
    rows = hkv * total
    if case["kind"] == "cache":
        cache = rows * 2 * d * es
    else:
        g = case["group"]
        cache = rows * (d + 8 * (d // g)) + 8 * d * hkv * sum(-(-n // g) for n in lens)
    return {"bytes": cache + small, "flops": 4 * d * hq * (total + tails)}
