"""The operators that bring prompts into the paged KV cache and read what requests share in it, and
the cases that they are measured on.

A case is a dict of plain values.  Its ``kind``:

* ``append``   queries, keys and values of new tokens as the products leave them: queries and keys
               normalised per head and rotated by their positions, keys and values written into the
               paged cache (``RopeAppendPlan``);
* ``prefill``  causal attention of packed new tokens over a paged cache that already holds their keys
               and values, and those of the positions before them (``PrefillPlan``);
* ``shared``   decode attention of one query per request where groups of requests share a prefix: the
               prefix's pages once for the whole group, then each request's own pages
               (``SharedDecodePlan``).

``own`` selects between the framework's operators and their plain forms: elementary torch operations
in 32 bits (angles in 64), rounded once at the end.
"""

import math
import random

import torch

own = False

D, P = 128, 16          # head dimension and page size, the library's own
SCALE = 1.0 / math.sqrt(D)
EPS = 1e-6
THETA = 1e6


def _append(name, requests=1, hq=16, hkv=8, tokens=1, ctx=0, layout="half", rotary=128, norm=True,
            stretch=1.0, fused=True):
    """``tokens``: new tokens of the longest request (1: one each, a decode step; else log-uniform
    below it); ``ctx``: cached positions of the longest request; ``rotary``: rotated dims of a head;
    ``stretch``: factor by which the context was extended (angles divided, cos and sin scaled);
    ``fused``: q, k and v are column slices of one product's output."""
    c = dict(kind="append", requests=requests, hq=hq, hkv=hkv, tokens=tokens, ctx=ctx, layout=layout,
             rotary=rotary, norm=norm, stretch=stretch, fused=fused)
    return dict(c, name=name) if name else c


def _prefill(name, requests=1, hq=16, hkv=8, tokens=512, ctx=0, sharp=1.0):
    """``tokens`` / ``ctx``: new tokens and cached positions of the longest request, the others'
    log-uniform below them; ``sharp``: factor on the queries (larger: a more peaked softmax)."""
    c = dict(kind="prefill", requests=requests, hq=hq, hkv=hkv, tokens=tokens, ctx=ctx, sharp=sharp)
    return dict(c, name=name) if name else c


def _shared(name, requests=32, groups=1, hq=16, hkv=8, prefix=8192, ctx=1024, shards=4, sharp=1.0):
    """``prefix``: shared positions of the first group (the others' log-uniform below them);
    ``ctx``: positions of its own that the longest request has; ``shards``: that they are cut into."""
    c = dict(kind="shared", requests=requests, groups=groups, hq=hq, hkv=hkv, prefix=prefix, ctx=ctx,
             shards=shards, sharp=sharp)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One request's decode step (Qwen3-0.6B heads, the 4,608-position context): pure latency.
        _append("append_b1_t1", ctx=4608),
        # A decode step of a full batch at Qwen3-4B's heads, far positions.
        _append("append_b64_t1_far", requests=64, hq=32, ctx=131071),
        # A chunk of several prompts in a context extended fourfold, half of each head rotated,
        # pairs interleaved, q, k and v as separate products.
        _append("append_b5_prompts", requests=5, hq=32, tokens=2731, ctx=9000, layout="interleaved",
                rotary=64, stretch=4.0, fused=False),
        # A long prompt at Qwen3-32B's heads: the largest amount of bytes.
        _append("append_b2_long", requests=2, hq=64, tokens=16384, ctx=1000),
        # A one-line prompt: latency.
        _prefill("prefill_b1_t37", tokens=37),
        # A few drafted tokens per request checked against long caches: bytes, few rows.
        _prefill("prefill_b4_t8_n36480", requests=4, hq=32, tokens=8, ctx=36480, sharp=2.0),
        # One prompt of 4,608 tokens at Qwen3-0.6B's heads.
        _prefill("prefill_b1_t4608", tokens=4608),
        # Packed prompts of mixed odd lengths at Qwen3-4B's heads, some with cached positions.
        _prefill("prefill_b8_ragged_g4", requests=8, hq=32, tokens=4099, ctx=777, sharp=2.0),
        # A chunk of a long prompt at Qwen3-32B's heads: the most matrix work.
        _prefill("prefill_b1_t4096_n12288_g8", hq=64, tokens=4096, ctx=12288),
        # A handful of chats over a short common instruction: latency.
        _shared("shared_b4_n1531", requests=4, prefix=1531, ctx=64, shards=1),
        # A serving batch over one long document, short chats of their own.
        _shared("shared_b32_n8192_g4", requests=32, hq=32, prefix=8192, ctx=1021, shards=4),
        # Many requests in three groups over long prefixes at Qwen3-32B's heads.
        _shared("shared_b128_n32768_g8", requests=128, groups=3, hq=64, prefix=32768, ctx=1999,
                shards=8, sharp=2.0),
    ]


MOST_SCORES = 3_600_000_000     # the plain form holds all scores of the padded batch at once


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "prefill", "shared"])
    hkv = rng.choice([2, 4, 8])
    hq = hkv * rng.choice([1, 2, 4, 8])
    if kind == "append":
        tokens = rng.choice([1, _log_int(rng, 2, 8000)])
        requests = _log_int(rng, 1, 256 if tokens == 1 else 8)
        return _append(None, requests, hq, hkv, tokens, _log_int(rng, 1, 131072),
                       rng.choice(["half", "interleaved"]), rng.choice([32, 64, 96, 128]),
                       rng.random() < 0.75, rng.choice([1.0, 4.0]), rng.random() < 0.5)
    if kind == "prefill":
        tokens = _log_int(rng, 1, 4096)
        ctx = min(_log_int(rng, 1, 65536), max(1, MOST_SCORES // (hq * tokens) - tokens))
        requests = _log_int(rng, 1, max(1, min(16, MOST_SCORES // (hq * tokens * (tokens + ctx)))))
        return _prefill(None, requests, hq, hkv, tokens, ctx, rng.choice([1.0, 2.0]))
    requests = _log_int(rng, 2, 128)
    prefix = _log_int(rng, 16, 32768)
    ctx = _log_int(rng, 1, 2000)
    return _shared(None, requests, rng.randint(1, min(4, requests)), hq, hkv, prefix, ctx,
                   max(1, ctx // 256), rng.choice([1.0, 2.0]))


# ------------------------------------------------------------------------------------------------
# sizes (of the case alone) and inputs (of the seed)
# ------------------------------------------------------------------------------------------------
def _spread(rng, longest, n):
    """n lengths: the longest first, the others log-uniform in [longest / 64, longest]."""
    return [longest] + [max(1, _log_int(rng, max(1, longest / 64), longest)) if longest else 0
                        for _ in range(n - 1)]


def _sizes(c):
    """Host integers of a case: new tokens (or group sizes), cached positions, prefix lengths."""
    rng = random.Random("%s" % sorted((k, v) for k, v in c.items() if k != "name"))
    n = c["requests"]
    if c["kind"] == "shared":
        cuts = sorted(rng.sample(range(1, n), c["groups"] - 1))
        return dict(rows=[0, *cuts, n], prefix=_spread(rng, c["prefix"], c["groups"]),
                    ctx=_spread(rng, c["ctx"], n))
    lens = [1] * n if c["tokens"] == 1 else _spread(rng, c["tokens"], n)
    return dict(lens=lens, ctx=_spread(rng, c["ctx"], n))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _table(gen, pages, width, first=None):
    """A block table of rows of ``pages`` entries at random places of a pool of just those pages
    (``first``: rows' entries start there), -1 where nothing is to be read; and the pool's size."""
    total = max(1, sum(pages))
    perm = torch.randperm(total, generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    table = torch.full((len(pages), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        lo = first[b] if first else 0
        table[b, lo:lo + n] = perm[at:at + n]
        at += n
    return table, total


def _pages(n):
    return -(-n // P)


def _normal(gen, *shape, scale=1.0):
    x = torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    return x.mul_(scale) if scale != 1.0 else x


def prepare(case, seed):
    c, z = case, _sizes(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    hq, hkv = c["hq"], c["hkv"]
    st = dict(case=c, ctx_lens=_ints(z["ctx"]))
    if c["kind"] == "append":
        lens, ctx = z["lens"], z["ctx"]
        T = sum(lens)
        first = [n // P for n in ctx]
        # Only the pages that this call writes are in the pool: those of the cached positions are
        # not touched by it.
        pages = [_pages(n + l) - f for n, l, f in zip(ctx, lens, first)]
        st["block_table"], pool = _table(gen, pages, max(f + n for f, n in zip(first, pages)), first)
        if c["fused"]:
            st["q"], st["k"], st["v"] = _normal(gen, T, (hq + 2 * hkv) * D).view(T, -1, D).split(
                [hq, hkv, hkv], 1)
        else:
            st["q"], st["k"], st["v"] = (_normal(gen, T, h, D) for h in (hq, hkv, hkv))
        for g in ("q_gain", "k_gain"):
            st[g] = (torch.rand(D, generator=gen, device="cuda") + 0.5).bfloat16() if c["norm"] else None
        half = torch.arange(0, c["rotary"], 2, dtype=torch.float64, device="cuda")
        st["freqs"] = THETA ** (-half / c["rotary"]) / c["stretch"]
        st["amplitude"] = 0.1 * math.log(c["stretch"]) + 1.0
        st["cu_tokens"] = _ints([0, *torch.tensor(lens).cumsum(0).tolist()])
        st["k_cache"], st["v_cache"] = (_normal(gen, pool, hkv, P, D) for _ in range(2))
        st["q_out"] = torch.empty((T, hq, D), dtype=torch.bfloat16, device="cuda")
        if own:
            import paper_2608_15473_amd as qf
            st["plan"] = qf.RopeAppendPlan(
                st["q"], st["k"], st["v"], st["k_cache"], st["v_cache"], st["block_table"],
                st["ctx_lens"], None if c["tokens"] == 1 else st["cu_tokens"], freqs=st["freqs"],
                layout=c["layout"], amplitude=st["amplitude"], q_gain=st["q_gain"],
                k_gain=st["k_gain"], eps=EPS, q_out=st["q_out"])
        return st
    if c["kind"] == "prefill":
        lens, ctx = z["lens"], z["ctx"]
        T, total = sum(lens), [n + l for n, l in zip(ctx, lens)]
        pages = [_pages(n) for n in total]
        st["block_table"], pool = _table(gen, pages, max(pages))
        st["longest"], st["positions"] = max(lens), max(total)
        st["q"] = _normal(gen, T, hq, D, scale=c["sharp"])
        st["cu_tokens"] = _ints([0, *torch.tensor(lens).cumsum(0).tolist()])
        rows = T
    else:
        rows = c["requests"]
        pages = [_pages(n) for n in z["prefix"]] + [_pages(n) for n in z["ctx"]]
        table, pool = _table(gen, pages, max(pages))
        st["prefix_table"] = table[:c["groups"], :max(pages[:c["groups"]])].contiguous()
        st["block_table"] = table[c["groups"]:, :max(pages[c["groups"]:])].contiguous()
        st["prefix_lens"], st["prefix_rows"] = _ints(z["prefix"]), _ints(z["rows"])
        st["n_shards"] = _ints([max(1, min(c["shards"], -(-n // 256))) for n in z["ctx"]])
        st["longest"] = max(b - a for a, b in zip(z["rows"], z["rows"][1:]))
        st["q"] = _normal(gen, rows, hq, D, scale=c["sharp"])
    st["k_cache"], st["v_cache"] = (_normal(gen, pool, hkv, P, D) for _ in range(2))
    if own:
        import paper_2608_15473_amd as qf
        if c["kind"] == "prefill":
            st["plan"] = qf.PrefillPlan(st["q"], st["k_cache"], st["v_cache"], st["block_table"],
                                        st["ctx_lens"], st["cu_tokens"], scale=SCALE)
        else:
            st["plan"] = qf.SharedDecodePlan(
                st["q"], st["k_cache"], st["v_cache"], st["prefix_table"], st["prefix_lens"],
                st["prefix_rows"], st["block_table"], st["ctx_lens"], st["n_shards"],
                max_shards=c["shards"], scale=SCALE)
    return st


# ------------------------------------------------------------------------------------------------
# the plain forms
# ------------------------------------------------------------------------------------------------
def _owner(starts, n):
    """For each of n rows, which range of ``starts`` it lies in, and its place there."""
    row = torch.arange(n, dtype=torch.int32, device="cuda")
    of = torch.searchsorted(starts, row, right=True) - 1
    return of, row - starts[of]


def _rms(x, gain):
    x = x.float()
    if gain is None:
        return x
    return x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * gain.float()


def _rotate(x, cos, sin, layout):
    r = 2 * cos.shape[-1]
    x, rest = x[..., :r], x[..., r:]
    if layout == "half":
        a, b = x[..., :r // 2], x[..., r // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _plain_append(st):
    c = st["case"]
    of, i = _owner(st["cu_tokens"], st["q"].shape[0])
    pos = (st["ctx_lens"][of] + i).long()
    angle = pos.double()[:, None] * st["freqs"]
    cos, sin = ((f(angle) * st["amplitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    st["q_out"].copy_(_rotate(_rms(st["q"], st["q_gain"]), cos, sin, c["layout"]))
    page = st["block_table"][of, pos // P].long()
    st["k_cache"][page, :, pos % P] = _rotate(_rms(st["k"], st["k_gain"]), cos, sin,
                                              c["layout"]).bfloat16()
    st["v_cache"][page, :, pos % P] = st["v"]
    return dict(q=st["q_out"], k_cache=st["k_cache"], v_cache=st["v_cache"])


def _paged(cache, table):
    """[rows, Hkv, positions, D] in 32 bits: the pages of each row of the table, in order."""
    x = cache[table.clamp(min=0).long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, D).float()


def _scores(q, k, lens):
    """q [rows, Hkv, queries, D] . k [rows, Hkv, n, D], -inf past each query's ``lens``
    ([rows, 1 or Hkv, queries, 1])."""
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(SCALE)
    at = torch.arange(k.shape[2], device="cuda", dtype=torch.int32)
    return s.masked_fill_(at >= lens, -math.inf)


def _plain_prefill(st):
    c, q, B = st["case"], st["q"], st["case"]["requests"]
    T, hq, hkv, L = q.shape[0], c["hq"], c["hkv"], st["longest"]
    of, i = _owner(st["cu_tokens"], T)
    padded = torch.zeros((B, L, hq, D), dtype=torch.float32, device="cuda")
    padded[of, i] = q.float()
    padded = padded.view(B, L, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, D)
    rows = torch.arange(L, device="cuda", dtype=torch.int32).repeat(hq // hkv)
    lens = (st["ctx_lens"][:, None] + rows + 1)[:, None, :, None]
    s = _scores(padded, _paged(st["k_cache"], st["block_table"]), lens)
    m = s.amax(-1, keepdim=True)
    s = s.sub_(m).exp_()
    z = s.sum(-1, keepdim=True)
    o = torch.matmul(s, _paged(st["v_cache"], st["block_table"])) / z
    back = lambda x: x.view(B, hkv, hq // hkv, L, -1).permute(0, 3, 1, 2, 4)[of, i]  # noqa: E731
    return dict(out=back(o).reshape(T, hq, D).bfloat16(), lse=back(m + z.log()).reshape(T, hq))


def _plain_shared(st):
    c, q = st["case"], st["q"]
    B, hq, hkv, NG, L = c["requests"], c["hq"], c["hkv"], c["groups"], st["longest"]
    G = hq // hkv
    of, i = _owner(st["prefix_rows"], B)
    grouped = torch.zeros((NG, L, hkv, G, D), dtype=torch.float32, device="cuda")
    grouped[of, i] = q.float().view(B, hkv, G, D)
    grouped = grouped.transpose(1, 2).reshape(NG, hkv, L * G, D)
    s = _scores(grouped, _paged(st["k_cache"], st["prefix_table"]),
                st["prefix_lens"].view(NG, 1, 1, 1))
    t = _scores(q.float().view(B, hkv, G, D), _paged(st["k_cache"], st["block_table"]),
                st["ctx_lens"].view(B, 1, 1, 1))
    back = lambda x: x.view(NG, hkv, L, G, -1).transpose(1, 2)[of, i]  # noqa: E731
    ms, mt = s.amax(-1, keepdim=True), t.amax(-1, keepdim=True)
    s, t = s.sub_(ms).exp_(), t.sub_(mt).exp_()
    zs, zt = back(s.sum(-1, keepdim=True)), t.sum(-1, keepdim=True)
    os = back(torch.matmul(s, _paged(st["v_cache"], st["prefix_table"])))
    ot = torch.matmul(t, _paged(st["v_cache"], st["block_table"]))
    ms = back(ms)
    m = torch.maximum(ms, mt)
    a, b = (ms - m).exp(), (mt - m).exp()
    z = a * zs + b * zt
    return dict(out=((a * os + b * ot) / z).reshape(B, hq, D).bfloat16(),
                lse=(m + z.log()).reshape(B, hq))


def run(state):
    if own:
        r = state["plan"]()
        if state["case"]["kind"] == "append":
            return dict(q=r, k_cache=state["k_cache"], v_cache=state["v_cache"])
        return dict(out=r[0], lse=r[1])
    return dict(append=_plain_append, prefill=_plain_prefill,
                shared=_plain_shared)[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its results in 64 bits
# ------------------------------------------------------------------------------------------------
def work(case):
    c, z = case, _sizes(case)
    hq, hkv = c["hq"], c["hkv"]
    if c["kind"] == "append":
        T = sum(z["lens"])
        return dict(bytes=T * (hq + 2 * hkv) * D * 2 * 2, flops=T * (hq + hkv) * D * 8)
    if c["kind"] == "prefill":
        T = sum(z["lens"])
        seen = sum(l * n + l * (l + 1) // 2 for n, l in zip(z["ctx"], z["lens"]))
        kept = sum(n + l for n, l in zip(z["ctx"], z["lens"]))
    else:
        T = c["requests"]
        kept = sum(z["prefix"]) + sum(z["ctx"])
        seen = sum(n * (b - a) for n, a, b in zip(z["prefix"], z["rows"], z["rows"][1:])) + sum(z["ctx"])
    return dict(bytes=T * hq * (D * 4 + 4) + kept * hkv * D * 4, flops=4 * hq * D * seen)


def _attend(q, k, v, last):
    """One request and KV head in 64 bits: q [r, D], k and v [n, D]; query j sees k[:last[j]]."""
    s = (q @ k.T) * SCALE
    s[torch.arange(k.shape[0], device="cuda")[None] >= last[:, None]] = -math.inf
    lse = torch.logsumexp(s, -1)
    return torch.exp(s - lse[:, None]) @ v, lse


def exact(case, seed):
    c, z = case, _sizes(case)
    st = prepare(case, seed)
    hq, hkv, G = c["hq"], c["hkv"], c["hq"] // c["hkv"]
    if c["kind"] == "append":
        kc, vc = st["k_cache"].double(), st["v_cache"].double()
        out, at, half = [], 0, c["rotary"] // 2
        perm = torch.arange(c["rotary"], device="cuda")
        if c["layout"] == "interleaved":    # dims of a head in the order first members, second members
            perm = torch.cat([perm[0::2], perm[1::2]])
        for b, (n, l) in enumerate(zip(z["ctx"], z["lens"])):
            pos = torch.arange(n, n + l, device="cuda")
            turn = torch.polar(torch.full((l, half), st["amplitude"], dtype=torch.float64, device="cuda"),
                               pos[:, None] * st["freqs"][None])

            def turned(x, gain):
                x = x[at:at + l].double()
                if gain is not None:
                    x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS) * gain.double()
                w = torch.complex(x[..., perm[:half]], x[..., perm[half:]]) * turn[:, None]
                y = x.clone()
                y[..., perm] = torch.cat([w.real, w.imag], -1)
                return y

            out.append(turned(st["q"], st["q_gain"]))
            page = st["block_table"][b, pos // P].long()
            kc[page, :, pos % P] = turned(st["k"], st["k_gain"])
            vc[page, :, pos % P] = st["v"][at:at + l].double()
            at += l
        return dict(q=torch.cat(out), k_cache=kc, v_cache=vc)

    def positions(cache, row, n):
        x = cache[row[:_pages(n)].long()].double()
        return x.transpose(0, 1).reshape(hkv, -1, D)[:, :n]

    T = st["q"].shape[0]
    out = torch.empty((T, hq, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((T, hq), dtype=torch.float64, device="cuda")
    if c["kind"] == "prefill":
        at = 0
        for b, (n, l) in enumerate(zip(z["ctx"], z["lens"])):
            k, v = (positions(st[x], st["block_table"][b], n + l) for x in ("k_cache", "v_cache"))
            last = n + 1 + torch.arange(l, device="cuda")
            for h in range(hq):
                out[at:at + l, h], lse[at:at + l, h] = _attend(
                    st["q"][at:at + l, h].double(), k[h // G], v[h // G], last)
            at += l
        return dict(out=out, lse=lse)
    for g, n in enumerate(z["prefix"]):
        pk, pv = (positions(st[x], st["prefix_table"][g], n) for x in ("k_cache", "v_cache"))
        for b in range(z["rows"][g], z["rows"][g + 1]):
            sk, sv = (positions(st[x], st["block_table"][b], z["ctx"][b]) for x in ("k_cache", "v_cache"))
            s = torch.matmul(st["q"][b].double().view(hkv, G, D),
                             torch.cat([pk, sk], 1).transpose(-1, -2)) * SCALE
            l = torch.logsumexp(s, -1, keepdim=True)
            out[b] = torch.matmul(torch.exp(s - l), torch.cat([pv, sv], 1)).view(hq, D)
            lse[b] = l.view(hq)
    return dict(out=out, lse=lse)
