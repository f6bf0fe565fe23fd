"""The performance cases of the paged softmax cache: what is measured.

A case is one pass through the entry points of
``paper_2607_24788_amd.paged`` (``prefill``, ``decode``, ``evict``): softmax
attention over a paged key-value cache, with a sliding window and a few first
tokens that stay visible (sinks), the attention weight that every cached token
has received, and the eviction of the tokens that received least.  With
``own`` false ``run`` computes the same in elementary torch operations, in 32
bits; ``exact`` gives it in 64 from the definition.

The definition, for query head h of KV head g = h // (Hq // Hkv), at position t
of a sequence of ``len`` cached tokens:
  visible(t) = {j <= t : j > t - W or j < n_sinks}
  out_t = sum_visible e^{tau q.k_j} v_j / sum_visible e^{tau q.k_j}
  lse_t = log sum_visible e^{tau q.k_j}
  weights_j += sum over the scored queries t and the heads of g of
               e^{tau q.k_j - lse_t}   (from 0 for a token that is new)
and an eviction keeps, per sequence and KV head, min(len, budget) tokens in
their order: the first n_sinks, the last n_recent, and of the others those of
the largest weights (of equal ones the first).

Fields of a case:
  op       "prefill": new tokens appended to the cache, one query each;
           "decode": one new token per sequence; "evict"
  batch, hq, hkv, d, dtype, page (tokens per page): the layer and its pages
  t_lo, t_hi   new tokens per sequence (prefill), or tokens cached (decode,
           with the new one; evict), spread over the batch
  history  tokens cached before a prefill
  window   W (0: every earlier token is visible), sinks
  observe  prefill: the last so many queries of each sequence are scored
  weights  decode: the step's attention weight is added up
  budget, recent, in_place   evict
"""
import math

import torch

own = False

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
FULL = 1 << 30   # a window that never ends

BASE = {"op": "prefill", "batch": 1, "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "page": 64, "t_lo": 8192,
        "t_hi": 8192, "history": 0, "window": 0, "sinks": 0, "observe": 0, "weights": False, "budget": 0, "recent": 0,
        "in_place": False}
SMALL = {"hq": 4, "hkv": 4, "d": 64, "dtype": "fp32", "page": 16}


def _case(name, **kw):
    c = dict(BASE, **kw)
    c["name"] = name
    return c


def listed():
    return [
        # the single fp32 layer: a prompt of 512 tokens, and a token after it
        # (launches and latency are all there is)
        _case("prefill_fp32_layer", t_lo=512, t_hi=512, window=64, sinks=4, **SMALL),
        _case("decode_fp32_layer", op="decode", t_lo=513, t_hi=513, window=64, sinks=4, **SMALL),
        # one chat session of an 8B-shaped model, 8K context: the prompt
        # through a layer with a window and sinks, and a token over all of it
        _case("prefill_8b_b1_w2048", window=2048, sinks=4),
        _case("decode_8b_b1", op="decode"),
        # a long prompt through a layer that keeps full attention
        _case("prefill_8b_32k", t_lo=32768, t_hi=32768),
        # chunked serving: odd numbers of new tokens onto 16K of history, the
        # last 32 queries scored for an eviction that follows
        _case("extend_8b_b8_w4000", batch=8, t_lo=301, t_hi=2047, history=16001, window=4000, sinks=4, observe=32,
              page=32),
        # a few drafted tokens per sequence, checked over a long cache
        _case("extend_8b_b4_draft", batch=4, t_lo=3, t_hi=9, history=32003),
        # a serving batch of 32 ragged sequences, 16K .. 32K tokens each
        _case("decode_8b_b32", op="decode", batch=32, t_lo=16384, t_hi=32768),
        # a 70B-shaped layer, an odd long window with sinks, weights added up
        _case("decode_70b_b8_weights", op="decode", batch=8, hq=64, t_lo=32768, t_hi=65536, window=8191, sinks=4,
              weights=True),
        # evictions: a small layer in place; a session's cache of 8K tokens
        # to 1024, and a batch's 16K .. 32K to 4096, into fresh pages
        _case("evict_fp32_layer", op="evict", batch=2, t_lo=450, t_hi=700, budget=257, recent=32, sinks=4,
              in_place=True, **SMALL),
        _case("evict_8b_b1", op="evict", budget=1024, recent=256, sinks=4),
        _case("evict_8b_b32", op="evict", batch=32, t_lo=16384, t_hi=32768, budget=4096, recent=1000, sinks=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A call of the same ranges (odd sizes among them)."""
    c = dict(BASE)
    c["op"] = rng.choice(["prefill", "prefill", "decode", "decode", "evict"])
    c["hq"], c["hkv"], c["d"] = rng.choice([(32, 8, 128), (32, 8, 128), (64, 8, 128), (8, 8, 128), (4, 4, 64),
                                            (24, 8, 64), (32, 2, 128)])
    c["batch"] = _log_int(rng, 1, 32)
    c["page"] = rng.choice([16, 32, 64, 64, 128, 256])
    if rng.random() < 0.2:
        c["dtype"] = "fp32"
    c["sinks"] = rng.choice([0, 4, rng.randint(1, 100)])
    small = 4 if c["dtype"] == "fp32" else 1  # fp32 holds a quarter
    if c["op"] == "prefill":
        c["window"] = 0 if rng.random() < 0.4 else _log_int(rng, 16, 8192)
        c["history"] = 0 if rng.random() < 0.4 else _log_int(rng, 16, 32768)
        c["t_hi"] = _log_int(rng, 1, 8192)
        c["observe"] = rng.choice([0, 0, 32, _log_int(rng, 1, 512)])
        # new tokens x keys x heads: at most a quarter of the longest prompt's
        most = (1 << 32) // small
        while c["batch"] > 1 and c["batch"] * c["t_hi"] * (c["history"] + c["t_hi"]) * c["hq"] > most:
            c["batch"] -= 1
        while c["t_hi"] > 1 and c["t_hi"] * (c["history"] + c["t_hi"]) * c["hq"] > most:
            c["t_hi"] = c["t_hi"] * 3 // 4
        c["history"] = min(c["history"], 393216 // c["batch"])
    else:
        c["t_hi"] = min(_log_int(rng, 16, 65536), 786432 // small // c["batch"])
        if c["op"] == "decode":
            c["window"] = 0 if rng.random() < 0.5 else _log_int(rng, 16, 16384)
            c["weights"] = rng.random() < 0.4
        else:
            c["recent"] = rng.randint(0, c["t_hi"] // 4)
            c["budget"] = c["sinks"] + c["recent"] + _log_int(rng, 1, max(2, c["t_hi"] // 2))
            c["in_place"] = rng.random() < 0.5
    c["t_lo"] = max(1, int(c["t_hi"] * rng.choice([0.5, 0.8, 1.0])))
    return c


# ---------------------------------------------------------------------------
# sizes

def _new(c):
    """New tokens per sequence, or tokens cached: spread evenly over [t_lo, t_hi] in a fixed mixed order."""
    B, lo, hi = c["batch"], c["t_lo"], c["t_hi"]
    if B == 1:
        return [hi]
    step = next(s for s in (5, 7, 3, 11, 13) if math.gcd(s, B) == 1)
    return [lo + round((hi - lo) * ((b * step) % B) / (B - 1)) for b in range(B)]


def _lens(c):
    """Tokens cached per sequence, the call's own new ones among them."""
    return [c["history"] + n if c["op"] == "prefill" else n for n in _new(c)]


def _window(c):
    return c["window"] or FULL


def _visible(c, p0, n):
    """sum over positions t in [p0, p0 + n) of the tokens that t sees."""
    W, s = _window(c), c["sinks"]
    t0, t1 = p0, p0 + n

    def upto(x, cap):  # sum over t in [t0, t1) of min(t + 1 - x, cap), where that is positive
        a, b = max(t0, x), max(t1, x)
        m = max(a, min(b, x + cap))      # below m: t + 1 - x
        return (m - a) * (a + 1 - x) + (m - a) * (m - a - 1) // 2 + (b - m) * cap
    # the window's tokens, and of the sinks those before it
    return upto(0, W) + (upto(W, s) if s else 0)


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    d, Hq, Hkv = c["d"], c["hq"], c["hkv"]
    row = 2 * Hkv * d * e                    # a token's K and V
    bytes_, flops = 0.0, 0.0
    for n, length in zip(_new(c), _lens(c)):
        if c["op"] == "evict":
            kept = min(length, c["budget"])
            bytes_ += 4 * Hkv * length + 2 * kept * row + kept * Hkv * (4 + 4)
            flops += Hkv * length
            continue
        n = 1 if c["op"] == "decode" else n
        p0 = length - n
        held = min(p0, _window(c) - 1)
        held += min(max(p0 - held, 0), c["sinks"])
        # held tokens read, new ones read and written to their pages, q in, out and lse out
        bytes_ += (held + 2 * n) * row + 2 * n * Hq * d * e + 4 * n * Hq
        flops += 4 * Hq * d * _visible(c, p0, n)
        scored = (1 if c["weights"] else 0) if c["op"] == "decode" else min(n, c["observe"])
        if scored:
            bytes_ += 8 * Hkv * (held + n)
            flops += 0 if c["op"] == "decode" else 2 * Hq * d * _visible(c, length - scored, scored)
    return {"bytes": bytes_, "flops": flops}


# ---------------------------------------------------------------------------
# inputs

def _inputs(c, seed):
    """Every tensor of the case, from its seed."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 29)
    dt, d, P, B, Hkv = DTYPE[c["dtype"]], c["d"], c["page"], c["batch"], c["hkv"]
    new, lens = _new(c), _lens(c)

    def normal(shape, scale):
        x = torch.empty(shape, dtype=dt, device="cuda")
        flat, step = x.view(-1), 1 << 28
        for i in range(0, flat.numel(), step):
            n = min(step, flat.numel() - i)
            flat[i:i + n] = torch.randn(n, generator=g, device="cuda").mul_(scale)
        return x

    def table(counts, first, wide):
        """Pages first .. of the pool, in mixed order; -1 behind a sequence's last."""
        n = sum(counts)
        ids = (torch.randperm(n, generator=g, device="cuda") + first).to(torch.int32)
        t = torch.full((B, wide), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, k in enumerate(counts):
            t[b, :k] = ids[at:at + k]
            at += k
        return t

    pages = [-(-n // P) for n in lens]
    x = {"max_pages": max(pages) + 1}
    dst = 0
    if c["op"] == "evict" and not c["in_place"]:
        dst = B * -(-c["budget"] // P)
    x["n_pages"] = sum(pages) + 3 + dst
    x["table"] = table(pages, 3, x["max_pages"])
    x["dst"] = table([-(-min(n, c["budget"]) // P) for n in lens], 3 + sum(pages), x["max_pages"]) if dst else None
    x["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    # scores of unit deviation, of 2 now and then: a few tokens of a row carry much of it
    x["k_pool"] = normal((x["n_pages"], Hkv, P, d), 1.0)
    x["v_pool"] = normal((x["n_pages"], Hkv, P, d), 1.0)
    if c["op"] == "evict":
        # what tokens have received: a few much, most little, the newest nothing yet (equal weights)
        w = torch.rand((x["n_pages"], Hkv, P), generator=g, device="cuda")
        x["w_pool"] = torch.where(w < 0.05, 0.0, w.pow(6) * 8)
        return x
    x["w_pool"] = None
    if c["weights"] or c["observe"]:
        x["w_pool"] = torch.rand((x["n_pages"], Hkv, P), generator=g, device="cuda")
    T = B if c["op"] == "decode" else sum(new)
    x["q"] = normal((T, c["hq"], d), 1.0 + (int(seed) % 2))
    x["k"] = normal((T, Hkv, d), 1.0)
    x["v"] = normal((T, Hkv, d), 1.0)
    return x


class State:
    pass


def prepare(case, seed):
    c = case
    x = _inputs(c, seed)
    st = State()
    st.c, st.lens_host, st.max_len = c, _lens(c), max(_lens(c))
    st.cu = [0]
    for n in _new(c):
        st.cu.append(st.cu[-1] + (1 if c["op"] == "decode" else n))
    for name, v in x.items():
        setattr(st, name, v)
    if c["op"] == "evict":
        st.kept = torch.empty((c["batch"], c["hkv"], c["budget"]), dtype=torch.int32, device="cuda")
        st.new_lens = torch.empty_like(x["lens"])
    else:
        st.out = torch.empty_like(x["q"])
        st.lse = torch.empty(x["q"].shape[:2], dtype=torch.float32, device="cuda")
    if own:
        from paper_2607_24788_amd import paged
        st.g = paged.Paged(c["batch"], c["hq"], c["hkv"], c["d"], c["page"], x["n_pages"], x["max_pages"],
                           window=_window(c), n_sinks=c["sinks"], dtype=DTYPE[c["dtype"]])
        st.cache = st.g.cache(x["k_pool"], x["v_pool"], x["table"], x["lens"], x["w_pool"])
        st.ws = st.g.new_workspace(st.cu[-1] if c["op"] == "prefill" else 0, weights=x["w_pool"] is not None)
    return st


# ---------------------------------------------------------------------------
# one pass

def run(state):
    st, c = state, state.c
    if c["op"] == "evict":
        if own:
            st.g.evict(st.cache, c["budget"], c["recent"], st.kept, st.new_lens, st.ws, dst_table=st.dst)
        else:
            st.kept, st.new_lens = _plain_evict(st)
        return [st.kept, st.new_lens, st.k_pool, st.v_pool, st.w_pool]
    if own and c["op"] == "decode":
        st.g.decode(st.cache, st.q, st.out, st.ws, k=st.k, v=st.v, lse=st.lse, max_len=st.max_len)
    elif own:
        st.g.prefill(st.cache, st.q, st.cu, st.out, st.ws, k=st.k, v=st.v, lse=st.lse, n_observe=c["observe"],
                     max_len=st.max_len)
    elif c["op"] == "decode":
        _plain_decode(st)
    else:
        _plain_prefill(st)
    return [st.out, st.lse, st.k_pool, st.v_pool] + ([st.w_pool] if st.w_pool is not None else [])


def _attend(c, q, k, v, see):
    """q [..][R][d], k, v [..][n][d] in fp32, see [..][R][n] -> out [..][R][d], lse [..][R], p [..][R][n]."""
    s = (q @ k.transpose(-1, -2)).mul_(c["d"] ** -0.5).masked_fill_(~see, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(total)
    return p @ v, (m + total.log()).squeeze(-1), p


def _see(c, t, n):
    """t [R] positions of queries -> [R][n]: the cached tokens that each sees."""
    j = torch.arange(n, device=t.device)
    t = t[:, None]
    return (j <= t) & ((j > t - _window(c)) | (j < c["sinks"]))


def _plain_prefill(st):
    c, P, Hkv, G, d = st.c, st.c["page"], st.c["hkv"], st.c["hq"] // st.c["hkv"], st.c["d"]
    for b, length in enumerate(st.lens_host):          # ragged: a sequence at a time
        i0, n = st.cu[b], st.cu[b + 1] - st.cu[b]
        p0 = length - n
        pos = torch.arange(p0, length, device="cuda")
        page = st.table[b][pos // P].long()
        st.k_pool[page, :, pos % P] = st.k[i0:i0 + n]
        st.v_pool[page, :, pos % P] = st.v[i0:i0 + n]
        held = st.table[b, :-(-length // P)].long()
        k = st.k_pool[held].transpose(0, 1).reshape(Hkv, -1, d).float()
        v = st.v_pool[held].transpose(0, 1).reshape(Hkv, -1, d).float()
        if c["observe"]:
            st.w_pool[page, :, pos % P] = 0.0
        step = max(1, (1 << 29) // (c["hq"] * length))   # scores of a block of queries: 2 GiB
        for a in range(0, n, step):
            e = min(n, a + step)
            m = p0 + e                                 # tokens up to the block's last
            q = st.q[i0 + a:i0 + e].float().view(e - a, Hkv, G, d).permute(1, 2, 0, 3).reshape(Hkv, G * (e - a), d)
            see = _see(c, pos[a:e], m).repeat(G, 1)
            o, lse, p = _attend(c, q, k[:, :m], v[:, :m], see)
            st.out[i0 + a:i0 + e] = o.view(Hkv, G, e - a, d).permute(2, 0, 1, 3).reshape(e - a, c["hq"], d)
            st.lse[i0 + a:i0 + e] = lse.view(Hkv * G, e - a).t()
            first = max(a, n - c["observe"])
            if first < e:
                w = p.view(Hkv, G, e - a, m)[:, :, first - a:].sum((1, 2))
                all_ = torch.arange(m, device="cuda")
                st.w_pool[held[all_ // P], :, all_ % P] += w.t()


def _plain_decode(st):
    c, P, Hkv, G, d = st.c, st.c["page"], st.c["hkv"], st.c["hq"] // st.c["hkv"], st.c["d"]
    B = c["batch"]
    t = st.lens.long() - 1
    page = st.table.gather(1, (t // P)[:, None])[:, 0].long()
    st.k_pool[page, :, t % P] = st.k
    st.v_pool[page, :, t % P] = st.v
    held = st.table[:, :-(-st.max_len // P)].long()
    k = st.k_pool[held.clamp_min(0)].transpose(1, 2).reshape(B, Hkv, -1, d).float()
    v = st.v_pool[held.clamp_min(0)].transpose(1, 2).reshape(B, Hkv, -1, d).float()
    see = _see(c, t, k.shape[2])[:, None, None, :]
    o, lse, p = _attend(c, st.q.float().view(B, Hkv, G, d), k, v, see)
    st.out.copy_(o.view(B, c["hq"], d))
    st.lse.copy_(lse.view(B, c["hq"]))
    if c["weights"]:
        st.w_pool[page, :, t % P] = 0.0
        b, i = torch.nonzero(held >= 0, as_tuple=True)
        st.w_pool[held[b, i]] += p.sum(2).view(B, Hkv, -1, P).transpose(1, 2)[b, i]


def _plain_evict(st):
    c, P, Hkv, B, budget = st.c, st.c["page"], st.c["hkv"], st.c["batch"], st.c["budget"]
    n = st.max_len
    j = torch.arange(n, device="cuda")
    held = st.table.long().clamp_min(0)
    w = st.w_pool[held[:, j // P], :, j % P].permute(0, 2, 1)             # [B][Hkv][n]
    length = st.lens.long()[:, None, None]
    key = w.masked_fill((j < c["sinks"]) | (j >= length - c["recent"]), math.inf).masked_fill(j >= length, -1.0)
    order = key.sort(dim=-1, descending=True, stable=True).indices[..., :budget]
    count = st.lens.clamp_max(budget)
    width = order.shape[-1]
    i = torch.arange(width, device="cuda")
    live = i < count[:, None, None]
    kept = order.masked_fill(~live, n).sort(dim=-1).values                    # the kept first, in their order
    to = st.table if st.dst is None else st.dst
    b, h, at = torch.nonzero(live.expand_as(kept), as_tuple=True)
    src = kept[b, h, at]
    sp, dp = held[b, src // P], to[b, at // P].long()
    for pool in (st.k_pool, st.v_pool, st.w_pool):
        pool[dp, h, at % P] = pool[sp, h, src % P]
    out = torch.full((B, Hkv, budget), -1, dtype=torch.int32, device="cuda")
    out[..., :width] = kept.masked_fill(~live, -1)
    return out, count


# ---------------------------------------------------------------------------
# the definition in 64 bits

def _rows(c, table_row, n):
    """Flat row of the pool, per KV head, of the first n tokens: [Hkv][n]."""
    j = torch.arange(n, device="cuda")
    page = table_row.long()[torch.div(j, c["page"], rounding_mode="floor")]
    head = torch.arange(c["hkv"], device="cuda")[:, None]
    return (page * c["hkv"] + head) * c["page"] + torch.remainder(j, c["page"])


def exact(case, seed):
    c = case
    x = _inputs(c, seed)
    k = x["k_pool"].view(-1, c["d"]).double()
    v = x["v_pool"].view(-1, c["d"]).double()
    w = x["w_pool"].view(-1).double() if x["w_pool"] is not None else None
    shape = x["k_pool"].shape
    lens = _lens(c)
    if c["op"] == "evict":
        return _exact_evict(c, x, k, v, w, shape)
    out = torch.zeros(x["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(x["q"].shape[:2], dtype=torch.float64, device="cuda")
    G, W, i0 = c["hq"] // c["hkv"], _window(c), 0
    for b, n in enumerate(lens):
        new = 1 if c["op"] == "decode" else _new(c)[b]
        rows = _rows(c, x["table"][b], n)
        for g in range(c["hkv"]):
            r = rows[g]
            k[r[n - new:]] = x["k"][i0:i0 + new, g].double()
            v[r[n - new:]] = x["v"][i0:i0 + new, g].double()
            scored = new if c["weights"] else min(new, c["observe"])
            if scored:
                w[r[n - new:]] = 0.0
            kg, vg = k[r], v[r]
            step = max(1, (1 << 26) // n)
            for h in range(g * G, (g + 1) * G):
                for a in range(0, new, step):
                    e = min(new, a + step)
                    t = torch.arange(n - new + a, n - new + e, device="cuda").view(-1, 1)
                    lo = 0 if c["sinks"] else max(0, n - new + a - W + 1)   # nothing before it is seen
                    j = torch.arange(lo, n - new + e, device="cuda").view(1, -1)
                    s = x["q"][i0 + a:i0 + e, h].double() @ kg[lo:n - new + e].t() / math.sqrt(c["d"])
                    hidden = torch.logical_or(j > t, torch.logical_and(t - j >= W, j >= c["sinks"]))
                    s[hidden] = -math.inf
                    z = torch.logsumexp(s, 1)
                    p = torch.exp(s - z[:, None])
                    out[i0 + a:i0 + e, h] = p @ vg[lo:n - new + e]
                    lse[i0 + a:i0 + e, h] = z
                    first = max(a, new - scored)
                    if first < e:
                        w[r[lo:n - new + e]] += p[first - a:].sum(0)
        i0 += new
    return [out, lse, k.view(shape), v.view(shape)] + ([w.view(shape[:3])] if w is not None else [])


def _exact_evict(c, x, k, v, w, shape):
    src_k, src_v, src_w = k.clone(), v.clone(), w.clone()
    dst = x["table"] if x["dst"] is None else x["dst"]
    kept = torch.full((c["batch"], c["hkv"], c["budget"]), -1, dtype=torch.int64, device="cuda")
    for b, n in enumerate(_lens(c)):
        m = min(n, c["budget"])
        rows, to = _rows(c, x["table"][b], n), _rows(c, dst[b], m)
        for g in range(c["hkv"]):
            r = rows[g]
            fixed = torch.zeros(n, dtype=torch.bool, device="cuda")
            fixed[:c["sinks"]] = True
            fixed[max(0, n - c["recent"]):] = True
            free = torch.nonzero(~fixed)[:, 0]
            more = max(0, m - int(fixed.sum()))
            best = torch.argsort(-src_w[r[free]], stable=True)[:more]
            keep = torch.sort(torch.cat([torch.nonzero(fixed)[:, 0], free[best]])).values[:m]
            kept[b, g, :m] = keep
            k[to[g]], v[to[g]], w[to[g]] = src_k[r[keep]], src_v[r[keep]], src_w[r[keep]]
    counts = torch.tensor([min(n, c["budget"]) for n in _lens(c)], device="cuda")
    return [kept, counts, k.view(shape), v.view(shape), w.view(shape[:3])]
