"""Norm + rotation + append, prefill and shared-prefix decode on the GPU against plain fp64 definitions.

Tolerances (derived before the first run):
  * rope_append: fp32 arithmetic on a pair of dims with products up to |x0| + |x1| in size and about ten
    roundings of 2^-24 (and an angle within 2^-22 rad): within DELTA_ROPE * (|x0| + |x1|) before the one
    rounding to bf16, so the output lies between the bf16 neighbours of the exact value less and plus that.
  * attention: the weights are rounded to bf16, each by at most 2^-8 of itself, so O moves by at most
    2^-8 sum w |v| / Z (``spread``); fp32 sums add far less (2^-14 of it allowed); then one rounding to
    bf16.  Over many outputs the roundings are independent: with iid normal values, 2^-8 / sqrt(3) of the
    norm each for the weights' and the output's own (2^-8 is their most), together below 2^-8 in norm.
  * log-sum-exp: 1e-5 * max(1, |LSE|), the library's gate.
"""

import numpy as np
import pytest
import torch

import paper_2608_15473_amd as qf
from oracle import prompt as oracle
from parity import bf16_neighbours

pytestmark = pytest.mark.gpu
SCALE = float(np.float32(128 ** -0.5))
DELTA_ROPE = 2.0 ** -20
WEIGHTS = 2.0 ** -8 + 2.0 ** -14
DEV = "cuda"


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def between(got, ref, delta, what=""):
    lo, _ = bf16_neighbours(ref - delta)
    _, hi = bf16_neighbours(ref + delta)
    ok = (got >= lo) & (got <= hi)
    assert ok.all(), (what, np.argwhere(~ok)[:4], got[~ok][:4], ref[~ok][:4])


def check_attention(out, lse, ref, norm=True, what=""):
    """Finite rows of the reference at the gates; NaN rows and empty ones exactly."""
    o, l = f64(out), f64(lse)
    O, L, spread = ref
    nan = np.isnan(L)
    assert np.isnan(l[nan]).all() and not np.isnan(l[~nan]).any(), what
    empty = L == -np.inf
    assert (l[empty] == -np.inf).all() and (o[empty] == 0).all(), what
    fine = ~nan & ~empty
    assert (np.abs(l[fine] - L[fine]) <= 1e-5 * np.maximum(1, np.abs(L[fine]))).all(), what
    values = fine[..., None] & np.isfinite(O)
    between(o[values], O[values], (WEIGHTS * spread)[values], what)
    assert (np.isnan(o) == np.isnan(O))[fine].all(), what
    if norm and values.sum() > 1000:
        err = np.linalg.norm((o - O)[values]) / np.linalg.norm(O[values])
        assert err <= 2.0 ** -8, (what, err)


def pool(gen, pages, hkv):
    return (torch.randn(pages, hkv, 16, 128, generator=gen).bfloat16() for _ in range(2))


def tables(gen, lens, width=None, spare=3):
    """Permuted block tables for the given position counts, -1 where nothing may be read."""
    need = [-(-n // 16) for n in lens]
    total = sum(need) + spare
    perm = torch.randperm(total, generator=gen).int()
    t = torch.full((len(lens), max([1, *need]) if width is None else width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = perm[at:at + n]
        at += n
    return t, total


def cu_of(lens):
    return torch.tensor([0, *np.cumsum(lens)], dtype=torch.int32)


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32)


# ------------------------------------------------------------------------------------------------
# norm, rotation, append
# ------------------------------------------------------------------------------------------------
def rope_case(seed, hq, hkv, lens, ctx, rotary=128, layout="half", norm=True, fused=False, amplitude=1.0,
              stretch=1.0, rows=0):
    gen = torch.Generator().manual_seed(seed)
    T = sum(lens) + rows                       # rows: of no request, at the end
    table, pages = tables(gen, [n + l for n, l in zip(ctx, lens)])
    kc, vc = pool(gen, pages, hkv)
    if fused:
        x = torch.randn(T, (hq + 2 * hkv) * 128 + 8, generator=gen).bfloat16().to(DEV)
        q, k, v = x[:, :-8].unflatten(1, (-1, 128)).split([hq, hkv, hkv], 1)
    else:
        q, k, v = (torch.randn(T, h, 128, generator=gen).bfloat16().to(DEV) for h in (hq, hkv, hkv))
    gains = [(torch.rand(128, generator=gen) + 0.5).bfloat16() if norm else None for _ in range(2)]
    freqs = qf.rope_frequencies(rotary, 1e6, stretch) if rotary else None
    return dict(q=q, k=k, v=v, kc=kc.to(DEV), vc=vc.to(DEV), table=table, ctx=ints(ctx), cu=cu_of(lens),
                gains=gains, freqs=freqs, layout=layout, amplitude=amplitude)


def run_rope(c, q_out=None, cu=True, **over):
    d = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    kw = dict(freqs=d(c["freqs"]), layout=c["layout"], amplitude=c["amplitude"], q_gain=d(c["gains"][0]),
              k_gain=d(c["gains"][1]), q_out=q_out)
    kw.update(over)
    return qf.qkv_rope_append(c["q"], c["k"], c["v"], c["kc"], c["vc"], d(c["table"]), d(c["ctx"]),
                              d(c["cu"]) if cu else None, **kw)


def rope_reference(c):
    return oracle.rope_append(f64(c["q"]), f64(c["k"]), f64(c["v"]), f64(c["kc"]), f64(c["vc"]),
                              c["table"].numpy(), c["ctx"].numpy(), c["cu"].numpy(),
                              gains=[f64(g) for g in c["gains"]],
                              freqs=None if c["freqs"] is None else c["freqs"].numpy(),
                              layout=c["layout"], amplitude=c["amplitude"])


def rope_delta(ref, c):
    """DELTA_ROPE times the pair's |x0| + |x1|, which sqrt(2) times its (unturned) length bounds."""
    r = 0 if c["freqs"] is None else len(c["freqs"])
    size = np.abs(ref)
    if r:
        pairs = ((np.arange(r), np.arange(r) + r) if c["layout"] == "half"
                 else (2 * np.arange(r), 2 * np.arange(r) + 1))
        size = size.copy()
        size[..., pairs[0]] = size[..., pairs[1]] = np.hypot(ref[..., pairs[0]], ref[..., pairs[1]]) * 2 ** 0.5
    return DELTA_ROPE * size


ROPE = [
    dict(hq=1, hkv=1, lens=[1], ctx=[0]),
    dict(hq=16, hkv=8, lens=[1, 1, 1], ctx=[0, 15, 4607]),
    dict(hq=32, hkv=8, lens=[5, 0, 17, 1], ctx=[12, 3, 0, 31], fused=True),
    dict(hq=8, hkv=1, lens=[33], ctx=[131040], layout="interleaved"),
    dict(hq=6, hkv=3, lens=[3, 20], ctx=[1048560, 5], rotary=64, layout="interleaved", fused=True),
    dict(hq=4, hkv=4, lens=[18], ctx=[999], rotary=96),
    dict(hq=2, hkv=2, lens=[7], ctx=[40], rotary=16, norm=False, amplitude=1.25, stretch=4.0),
    dict(hq=2, hkv=2, lens=[7], ctx=[40], rotary=0),
    dict(hq=2, hkv=1, lens=[9, 4], ctx=[2, 7], rotary=0, norm=False),
]


ROPE += [
    dict(hq=1, hkv=1, lens=[0] * 3 + [b % 3 for b in range(130)] + [0] * 70 + [2],
         ctx=[7 * b % 50 for b in range(204)]),
]


@pytest.mark.parametrize("kw", ROPE, ids=range(len(ROPE)))
def test_rope_append(gpu, kw):
    c = rope_case(11, **kw)
    ref_q, ref_k, ref_v = rope_reference(c)
    q = run_rope(c)
    between(f64(q), ref_q, rope_delta(ref_q, c), "q")
    between(f64(c["kc"]), ref_k, rope_delta(ref_k, c), "k")
    assert np.array_equal(f64(c["vc"]), ref_v)          # a copy, and nothing else written


def test_rope_decode_step_is_the_packed_call(gpu):
    """cu_tokens None is one token per request; queries in place; queries alone and keys alone."""
    kw = dict(seed=12, hq=16, hkv=4, lens=[1] * 70, ctx=[7 * b for b in range(70)])
    a, b, c = rope_case(**kw), rope_case(**kw), rope_case(**kw)
    qa, qb = run_rope(a), run_rope(b, q_out=b["q"], cu=False)
    assert qb is b["q"] and torch.equal(qa, qb) and torch.equal(a["kc"], b["kc"])
    assert torch.equal(a["vc"], b["vc"])
    before = c["kc"].clone()
    q, k, v = c["q"], c["k"], c["v"]
    c["k"] = c["v"] = None
    assert torch.equal(run_rope(c), qa) and torch.equal(c["kc"], before)
    c.update(q=None, k=k, v=v)
    assert run_rope(c) is None
    assert torch.equal(c["kc"], a["kc"]) and torch.equal(c["vc"], a["vc"])


def test_rope_rows_and_tokens_that_have_no_place(gpu):
    """Rows of no request are left alone; a token past the table or in a page outside the pool is not
    appended and sets the status; the queries of every token are written."""
    c = rope_case(13, 4, 2, [3, 20, 2], [14, 30, 0], rows=3)
    c["table"][1, 3] = c["kc"].shape[0]                 # positions 48, 49 of request 1
    c["ctx"][2] = c["table"].shape[1] * 16 - 1          # its second token is past the table
    c["table"][2, -1] = -7                              # and its first's page is none
    ref_q, ref_k, ref_v = rope_reference(c)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    q = torch.full((28, 4, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    run_rope(c, q_out=q, status=status)
    assert int(status) == 1
    between(f64(q)[:25], ref_q[:25], rope_delta(ref_q, c)[:25])
    assert bool((q[25:] == 7.0).all())
    between(f64(c["kc"]), ref_k, rope_delta(ref_k, c))
    assert np.array_equal(f64(c["vc"]), ref_v)
    ok = rope_case(13, 4, 2, [3, 20, 2], [14, 30, 0])
    status.zero_()
    run_rope(ok, status=status)
    assert int(status) == 0


def test_rope_index_arrays_out_of_order_stay_in_bounds(gpu):
    """Any contents of cu_tokens and ctx_lens: rows of requests that are out of order or range may be
    skipped, and nothing beside the caches and q_out changes."""
    for cu in ([0, 5, 3, 9], [-4, 2, 30, 9], [4, 4, 4, 4], [9, 9, 0, -1]):
        c = rope_case(14, 2, 1, [3, 3, 3], [0, 5, 20])
        c["cu"] = ints(cu)
        c["ctx"][1] = -3
        kc = c["kc"].clone()
        run_rope(c)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(c["kc"].float()).all()) and kc.shape == c["kc"].shape


# ------------------------------------------------------------------------------------------------
# prefill
# ------------------------------------------------------------------------------------------------
def prefill_case(seed, hq, hkv, lens, ctx, sharp=1.0, width=None, rows=0, garbage=True):
    gen = torch.Generator().manual_seed(seed)
    total = [n + l for n, l in zip(ctx, lens)]
    table, pages = tables(gen, total, width)
    kc, vc = pool(gen, pages, hkv)
    q = (torch.randn(sum(lens) + rows, hq, 128, generator=gen) * sharp).bfloat16()
    if garbage:                                # what the pool holds past a request's last position
        for b, n in enumerate(total):
            if n % 16:
                kc[table[b, n // 16], :, n % 16:] = float("nan")
                vc[table[b, n // 16], :, n % 16:] = float("inf")
    return dict(q=q, kc=kc, vc=vc, table=table, ctx=ints(ctx), cu=cu_of(lens), scale=SCALE)


def run_prefill(c, **kw):
    d = {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    return qf.attn_prefill(d["q"], d["kc"], d["vc"], d["table"], d["ctx"], d["cu"], scale=c["scale"], **kw)


def prefill_reference(c):
    return oracle.prefill(f64(c["q"]), f64(c["kc"]), f64(c["vc"]), c["table"].numpy(), c["ctx"].numpy(),
                          c["cu"].numpy(), c["scale"])


PREFILL = [
    dict(hq=1, hkv=1, lens=[1], ctx=[0]),
    dict(hq=2, hkv=1, lens=[1, 1, 1, 1], ctx=[0, 15, 16, 63]),
    dict(hq=8, hkv=1, lens=[17], ctx=[47]),
    dict(hq=16, hkv=2, lens=[3, 0, 16, 1], ctx=[64, 9, 0, 300]),
    dict(hq=4, hkv=1, lens=[65], ctx=[63]),
    dict(hq=4, hkv=4, lens=[130], ctx=[0]),
    dict(hq=2, hkv=1, lens=[64, 1, 127], ctx=[1, 65, 0], sharp=4.0),
    dict(hq=3, hkv=3, lens=[5, 129], ctx=[2000, 31], sharp=2.0),
    dict(hq=8, hkv=2, lens=[70, 3], ctx=[1000, 5003], sharp=2.0),        # key ranges
    dict(hq=1, hkv=1, lens=[2], ctx=[9000], width=4096),                 # a long table, many ranges
    dict(hq=64, hkv=8, lens=[2], ctx=[100]),
]


PREFILL += [
    dict(hq=4, hkv=2, lens=[3, 0, 40], ctx=[2, 0, 6000], sharp=2.0),     # one tile cut, others not
    dict(hq=1, hkv=1, lens=[1 + b % 2 for b in range(100)], ctx=[3000 if b == 77 else b for b in range(100)]),
    dict(hq=32, hkv=4, lens=[33], ctx=[2500], sharp=2.0),                # full tiles, cut
    dict(hq=8, hkv=1, lens=[1], ctx=[13000], sharp=2.0),                 # hundreds of ranges
]


@pytest.mark.parametrize("kw", PREFILL, ids=range(len(PREFILL)))
def test_prefill(gpu, kw):
    c = prefill_case(21, **kw)
    out, lse = run_prefill(c)
    check_attention(out, lse, prefill_reference(c))


def test_prefill_many_tiles(gpu):
    """Enough row tiles that no key ranges are made: requests of 0 to 90 tokens, G = 4, and one of G = 1
    heads long enough for several tiles."""
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 12, 300)]
    lens[7], lens[120] = 90, 41
    c = prefill_case(22, 4, 1, lens, [int(x) for x in rng.integers(0, 40, 300)], sharp=2.0)
    out, lse = run_prefill(c)
    check_attention(out, lse, prefill_reference(c))


def test_prefill_hundreds_of_requests(gpu):
    """More requests than a workgroup has threads: tiles of 1 to 128 steps in order of length, one request
    with a context that no table holds, another without rows; and few rows in all, whose keys are cut."""
    lens = [1 + 7 * b % 5 for b in range(600)]
    ctx = [61 * b % 257 for b in range(600)]
    lens[3], lens[299], ctx[299], ctx[411], lens[599] = 0, 75, 130, 8100, 140
    c = prefill_case(37, 2, 1, lens, ctx, sharp=2.0)
    ref = prefill_reference(c)
    c["ctx"][298] = c["table"].shape[1] * 16
    at = sum(lens[:298])
    for x in ref:
        x[at:at + lens[298]] = np.nan
    check_attention(*run_prefill(c), ref)
    c = prefill_case(38, 1, 1, [1 + (b == 280) for b in range(300)], [4000 if b == 280 else b for b in range(300)])
    check_attention(*run_prefill(c), prefill_reference(c))


def test_prefill_hundreds_of_row_ranges_out_of_order_stay_in_bounds(gpu):
    c = prefill_case(39, 2, 1, [3] * 300, [b % 70 for b in range(300)])
    c["cu"] = ints(np.random.default_rng(6).integers(-5, 905, 301))
    out, _ = run_prefill(c)
    torch.cuda.synchronize()
    assert out.shape == (900, 2, 128)


def test_pages_past_four_gibibytes(gpu):
    """A pool of which K alone is 5 GB, the pages at its end: appended to, read by prefill and as a prefix."""
    pages = 1_220_000
    c = prefill_case(40, 4, 1, [9, 40], [70, 0], garbage=False)
    d = {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    small = d["kc"].shape[0]
    far = dict(d, table=torch.where(d["table"] >= 0, d["table"] + (pages - small), d["table"]))
    for x in ("kc", "vc"):
        far[x] = torch.empty(pages, 1, 16, 128, dtype=torch.bfloat16, device=DEV)
        far[x][-small:] = d[x]
    new = torch.randn(49, 1, 128, generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    res = []
    for e in (d, far):
        qf.qkv_rope_append(None, new, new, e["kc"], e["vc"], e["table"], e["ctx"], e["cu"])
        res.append(qf.attn_prefill(e["q"], e["kc"], e["vc"], e["table"], e["ctx"], e["cu"]))
        res.append(qf.attn_decode_shared(e["q"][:2], e["kc"], e["vc"], e["table"][:1], e["ctx"][:1],
                                         ints([0, 2]).to(DEV), e["table"][1:].repeat(2, 1),
                                         ints([40, 3]).to(DEV), 1))
    for a, b in zip(res[0] + res[1], res[2] + res[3]):
        assert bool(torch.isfinite(a.float()).all()) and torch.equal(a, b)


def test_prefill_long_prompt(gpu):
    """Several hundred workgroups, one request: rows of every tile against fp64 (on the GPU, in torch)."""
    gen = torch.Generator().manual_seed(23)
    n, hq, hkv = 2333, 16, 8
    table, pages = tables(gen, [n])
    kc, vc = pool(gen, pages, hkv)
    q = torch.randn(n, hq, 128, generator=gen).bfloat16()
    out, lse = run_prefill(dict(q=q, kc=kc, vc=vc, table=table, ctx=ints([0]), cu=ints([0, n]), scale=SCALE))
    k, v = (c[table[0].long()].transpose(0, 1).reshape(hkv, -1, 128)[:, :n].double().to(DEV)
            for c in (kc, vc))
    for h in range(hq):
        s = q[:, h].double().to(DEV) @ k[h // 2].T * SCALE
        s.masked_fill_(torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1), -float("inf"))
        w = s.softmax(-1)
        ref = (f64(w @ v[h // 2]), f64(s.logsumexp(-1)), f64(w @ v[h // 2].abs()))
        check_attention(out[:, h], lse[:, h], ref, what=h)


@pytest.mark.parametrize("scale", [-SCALE, 0.0, 1.0, 12.0])
def test_prefill_scales(gpu, scale):
    """Negative, zero and large scales (logits of hundreds: one key takes nearly all the weight)."""
    c = prefill_case(24, 4, 2, [70, 9], [3, 80])
    c["scale"] = scale
    out, lse = run_prefill(c)
    check_attention(out, lse, prefill_reference(c), norm=abs(scale) < 1.0)


def test_prefill_nan_and_inf_stay_where_they_are_seen(gpu):
    """A NaN or infinite key or value reaches exactly the rows that see its position."""
    c = prefill_case(25, 4, 2, [150], [10], garbage=False)
    place = lambda pos: (int(c["table"][0, pos // 16]), 0, pos % 16)  # noqa: E731
    c["vc"][place(100)][5] = float("inf")
    c["vc"][place(101)][6] = -float("inf")
    c["vc"][place(130)][7] = float("nan")
    c["kc"][place(140)][:] = float("nan")
    c["kc"][place(150)][:] = float("inf")
    with np.errstate(invalid="ignore"):
        ref = prefill_reference(c)
    out, lse = run_prefill(c)
    check_attention(out, lse, ref, norm=False)
    o = f64(out)
    seen = np.arange(150) + 10
    for h in (0, 1):
        assert (o[(seen >= 100) & (seen < 140), h, 5] == np.inf).all()
        assert (o[(seen >= 101) & (seen < 140), h, 6] == -np.inf).all()
    assert np.isfinite(o[:, 2:]).all() and np.isfinite(o[seen < 100]).all()


def test_prefill_scores_of_minus_infinity(gpu):
    """Keys whose scores are -inf weigh nothing; a row that sees only such keys is empty."""
    c = prefill_case(26, 1, 1, [40], [0])
    c["q"] = c["q"].abs() + 0.1
    pos = lambda n: (int(c["table"][0, n // 16]), 0, n % 16)  # noqa: E731
    for n in (0, 1, 20):
        c["kc"][pos(n)][:] = -float("inf")
    with np.errstate(invalid="ignore"):
        ref = prefill_reference(c)
    assert np.isneginf(ref[1][:2]).all() and np.isfinite(ref[1][2:]).all()
    out, lse = run_prefill(c)
    check_attention(out, lse, ref)


def test_prefill_lowest_and_highest_finite_values(gpu):
    c = prefill_case(27, 2, 1, [40], [0])
    big = torch.finfo(torch.bfloat16).max
    pos = lambda n: (int(c["table"][0, n // 16]), 0, n % 16)  # noqa: E731
    c["q"].fill_(0.0)
    c["q"][:, :, 0] = 1.0
    c["kc"][pos(3)][0] = -big                  # a score of about -3e37
    c["kc"][pos(0)][0] = -big
    c["vc"][pos(17)][:] = big / 64
    out, lse = run_prefill(c)
    check_attention(out, lse, prefill_reference(c), norm=False)


def test_prefill_out_of_range_values_poison_their_request(gpu):
    """A context past the table, a negative one, a page outside the pool: NaN for the rows that see them,
    the other requests untouched; rows of no request left as they were."""
    c = prefill_case(28, 4, 2, [20, 30, 25, 9], [0, 10, 30, 5], rows=6)
    clean = prefill_reference(c)
    c["ctx"][0] = c["table"].shape[1] * 16 - 19
    c["ctx"][3] = -1
    c["table"][2, 2] = c["kc"].shape[0] + 5            # positions 32 .. 47 of request 2
    out = torch.full((90, 4, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((90, 4), 7.0, dtype=torch.float32, device=DEV)
    run_prefill(c, out=out, lse=lse)
    ref = [x.copy() for x in clean]
    bad = np.r_[0:20, 52:75, 75:84]                    # request 2's rows from position 32 on
    for x in ref:
        x[bad] = np.nan
    check_attention(out[:84], lse[:84], [x[:84] for x in ref])
    assert np.isnan(f64(out)[bad]).all()
    assert bool((out[84:] == 7.0).all()) and bool((lse[84:] == 7.0).all())


def test_prefill_row_ranges_out_of_order_stay_in_bounds(gpu):
    for cu in ([0, 9, 4, 12], [-2, 3, 6, 50], [12, 12, 12, 12], [3, 5, 5, 9]):
        c = prefill_case(29, 2, 1, [4, 4, 4], [40, 3, 900])
        c["cu"] = ints(cu)
        out = torch.full((12, 2, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        run_prefill(c, out=out)
        torch.cuda.synchronize()
        if cu == [3, 5, 5, 9]:
            assert bool((out[:3] == 7.0).all()) and bool((out[9:] == 7.0).all())
            assert not bool((out[3:9] == 7.0).all())


def test_a_table_has_the_pages_that_are_named(gpu):
    c = prefill_case(30, 4, 1, [2], [20])
    d = {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    wrong = d["table"].shape[1] + 1
    cache = (d["kc"], d["vc"], d["table"], d["ctx"])
    q = d["q"][:1]
    with pytest.raises(qf.QFError, match="pages a row"):
        qf.attn_prefill(d["q"], *cache, d["cu"], max_pages=wrong)
    with pytest.raises(qf.QFError, match="pages a row"):
        qf.qkv_rope_append(q, q[:, :1], q[:, :1], *cache, max_pages=wrong)
    with pytest.raises(qf.QFError, match="pages a row"):
        qf.attn_decode_shared(q, d["kc"], d["vc"], d["table"], d["ctx"], ints([0, 1]).to(DEV), d["table"],
                              d["ctx"], 1, max_pages=wrong)


def test_prefill_identity_table_and_no_lse(gpu):
    c = prefill_case(30, 4, 1, [9, 30], [20, 7], garbage=False)
    width = c["table"].shape[1]
    kc, vc = (torch.zeros(2 * width, 1, 16, 128, dtype=torch.bfloat16) for _ in range(2))
    for b in range(2):
        n = int((c["table"][b] >= 0).sum())
        for x, y in ((kc, c["kc"]), (vc, c["vc"])):
            x[b * width:b * width + n] = y[c["table"][b, :n].long()]
    a, la = run_prefill(c)
    d = dict(c, kc=kc, vc=vc)
    b_, lb = qf.attn_prefill(d["q"].to(DEV), kc.to(DEV), vc.to(DEV), None, d["ctx"].to(DEV),
                             d["cu"].to(DEV), scale=SCALE)
    assert torch.equal(a, b_) and torch.equal(la, lb)
    e, none = run_prefill(c, want_lse=False)
    assert none is None and torch.equal(a, e)


def test_prefill_agrees_with_the_decode_sweep(gpu):
    """The last row of a prompt is the decode step over all its positions."""
    c = prefill_case(31, 32, 8, [1, 1, 1], [100, 2047, 6000])
    out, lse = run_prefill(c)
    d = {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    o2, l2 = qf.attn_decode(d["q"], d["kc"], d["vc"], d["table"], d["ctx"] + 1, 4, scale=SCALE)
    assert (lse - l2).abs().max() <= 2e-5 * l2.abs().max()
    assert (out.float() - o2.float()).norm() <= 2.0 ** -7 * o2.float().norm()


# ------------------------------------------------------------------------------------------------
# shared prefixes
# ------------------------------------------------------------------------------------------------
def shared_case(seed, hq, hkv, rows, prefix, ctx, shards=2, sharp=1.0, garbage=True):
    gen = torch.Generator().manual_seed(seed)
    t, pages = tables(gen, [*prefix, *ctx])
    kc, vc = pool(gen, pages, hkv)
    if garbage:
        for b, n in enumerate([*prefix, *ctx]):
            if n % 16:
                kc[t[b, n // 16], :, n % 16:] = float("nan")
                vc[t[b, n // 16], :, n % 16:] = float("nan")
    ng = len(prefix)
    q = (torch.randn(len(ctx), hq, 128, generator=gen) * sharp).bfloat16()
    return dict(q=q, kc=kc, vc=vc, pt=t[:ng].contiguous(), pl=ints(prefix), rows=ints(rows),
                table=t[ng:].contiguous(), ctx=ints(ctx), ns=ints([shards] * len(ctx)), shards=shards)


def run_shared(c, **kw):
    d = {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    return qf.attn_decode_shared(d["q"], d["kc"], d["vc"], d["pt"], d["pl"], d["rows"], d["table"],
                                 d["ctx"], d["ns"], max_shards=c["shards"], scale=SCALE, **kw)


def shared_reference(c):
    return oracle.decode_shared(f64(c["q"]), f64(c["kc"]), f64(c["vc"]), c["pt"].numpy(), c["pl"].numpy(),
                                c["rows"].numpy(), c["table"].numpy(), c["ctx"].numpy(), SCALE)


SHARED = [
    dict(hq=1, hkv=1, rows=[0, 1], prefix=[1], ctx=[0]),
    dict(hq=16, hkv=8, rows=[0, 4], prefix=[100], ctx=[1, 0, 17, 64]),
    dict(hq=8, hkv=1, rows=[0, 17], prefix=[333], ctx=[5 * b for b in range(17)], sharp=2.0),
    dict(hq=4, hkv=1, rows=[0, 40], prefix=[65], ctx=[3] * 40),
    dict(hq=4, hkv=2, rows=[1, 3, 3, 8], prefix=[50, 20, 1000], ctx=[7, 0, 3, 90, 0, 31, 2, 8, 700, 0],
         shards=3, sharp=2.0),
    dict(hq=8, hkv=2, rows=[0, 2, 5], prefix=[0, 16], ctx=[0, 3, 0, 40, 1], shards=1),
    dict(hq=2, hkv=2, rows=[0, 2], prefix=[9001], ctx=[11, 2000], shards=7),
    dict(hq=2, hkv=1, rows=[2, 2], prefix=[64], ctx=[5, 0, 33]),               # nobody shares it
]


SHARED += [
    dict(hq=2, hkv=1, rows=[*range(71)], prefix=[1500 if i == 66 else 5 * i for i in range(70)],
         ctx=[b % 9 for b in range(71)], shards=1),
    dict(hq=16, hkv=2, rows=[0, 20, 90], prefix=[3000, 700], ctx=[7 * b % 41 for b in range(90)], sharp=2.0),
]


@pytest.mark.parametrize("kw", SHARED, ids=range(len(SHARED)))
def test_shared(gpu, kw):
    c = shared_case(41, **kw)
    out, lse = run_shared(c)
    check_attention(out, lse, shared_reference(c))


def test_shared_without_groups_is_the_plain_decode(gpu):
    c = shared_case(42, 4, 2, [0], [], [5, 700, 0, 33], shards=3)
    c["pt"] = torch.zeros(0, 1, dtype=torch.int32)
    out, lse = run_shared(c)
    check_attention(out, lse, shared_reference(c))


def test_shared_pair_takes_the_current_token(gpu):
    """pair=True is one slot of the merges that fold in (and append) the current token."""
    c = shared_case(43, 8, 2, [0, 3], [200], [16, 0, 45, 7], garbage=False)
    gen = torch.Generator().manual_seed(44)
    k, v = (torch.randn(4, 2, 128, generator=gen).bfloat16() for _ in range(2))
    po, pl = run_shared(c, pair=True)
    assert po.shape == (4, 1, 8, 128) and po.dtype == torch.float32
    out, lse = qf.attn_combine_current(po, pl, c["q"].to(DEV), k.to(DEV), v.to(DEV), scale=SCALE)
    # the reference: one more position of each request's own
    t2, pages = tables(gen, [200, *(int(n) + 1 for n in c["ctx"])])
    kc, vc = (torch.zeros(pages, 2, 16, 128) for _ in range(2))
    for row, n in enumerate([200, *map(int, c["ctx"])]):
        src = c["pt"][0] if row == 0 else c["table"][row - 1]
        for j in range(-(-n // 16)):
            kc[t2[row, j]], vc[t2[row, j]] = c["kc"][src[j]].float(), c["vc"][src[j]].float()
        if row:
            kc[t2[row, n // 16], :, n % 16] = k[row - 1].float()
            vc[t2[row, n // 16], :, n % 16] = v[row - 1].float()
    ref = oracle.decode_shared(f64(c["q"]), f64(kc), f64(vc), t2[:1].numpy(), np.array([200]),
                               c["rows"].numpy(), t2[1:].numpy(), c["ctx"].numpy() + 1, SCALE)
    check_attention(out, lse, ref)


def test_shared_out_of_range_values_poison_their_group(gpu):
    c = shared_case(45, 4, 2, [0, 2, 4, 6], [40, 50, 60], [3, 9, 20, 0, 8, 8, 4], garbage=False)
    ref = [x.copy() for x in shared_reference(c)]
    c["pl"][0] = c["pt"].shape[1] * 16 + 1
    c["pt"][2, 1] = -1
    c["ctx"][2] = -4
    for x in ref:
        x[[0, 1, 2, 4, 5]] = np.nan
    out, lse = run_shared(c)
    check_attention(out, lse, ref)
    assert np.isnan(f64(out)[[0, 1, 2, 4, 5]]).all()


# ------------------------------------------------------------------------------------------------
# together, streams, graphs
# ------------------------------------------------------------------------------------------------
def test_prompts_then_shared_decode(gpu):
    """A serving program's run of them: a common prompt written and attended once, each request's own
    tokens in a second chunk, then decode steps over the shared prefix; every attention against fp64 of
    the bytes in the cache, and the rotated queries against the definition."""
    hq, hkv, common, own, steps = 8, 2, 53, [5, 0, 21], 3
    gen = torch.Generator().manual_seed(51)
    dev = lambda t: t.to(DEV)  # noqa: E731
    freqs = dev(qf.rope_frequencies(128, 1e4))
    gains = [dev((torch.rand(128, generator=gen) + 0.5).bfloat16()) for _ in range(2)]
    table, pages = tables(gen, [64, *(64 + n + steps for n in own)])
    kc, vc = (dev(torch.full((pages, hkv, 16, 128), float("nan"), dtype=torch.bfloat16)) for _ in range(2))
    rand = lambda *s: dev(torch.randn(*s, generator=gen).bfloat16())  # noqa: E731

    def enter(tokens, tbl, ctx, cu):
        q, k, v = rand(tokens, hq, 128), rand(tokens, hkv, 128), rand(tokens, hkv, 128)
        got = qf.qkv_rope_append(q, k, v, kc, vc, dev(tbl), dev(ctx), None if cu is None else dev(cu),
                                 freqs=freqs, q_gain=gains[0], k_gain=gains[1])
        bounds = (cu if cu is not None else torch.arange(tokens + 1)).numpy()
        ref, _, _ = oracle.rope_append(f64(q), f64(k), f64(v), f64(kc), f64(vc), tbl.numpy(), ctx.numpy(),
                                       bounds, gains=[f64(g) for g in gains], freqs=f64(freqs))
        between(f64(got), ref, rope_delta(ref, dict(freqs=freqs, layout="half")))
        return got

    one = table[:1].contiguous()
    q = enter(common, one, ints([0]), ints([0, common]))
    out, lse = qf.attn_prefill(q, kc, vc, dev(one), dev(ints([0])), dev(ints([0, common])))
    check_attention(out, lse, oracle.prefill(f64(q), f64(kc), f64(vc), one.numpy(), [0], [0, common], SCALE))

    # Requests share the prefix's whole pages; what is past them is copied to a page of their own, and
    # their tables name the shared pages first, so that positions stay what they are.
    whole = common // 16
    for b in range(3):
        kc[int(table[1 + b, whole])], vc[int(table[1 + b, whole])] = kc[int(one[0, whole])], vc[int(one[0, whole])]
    full = torch.cat([one[:, :whole].expand(3, -1), table[1:, whole:]], 1).contiguous()
    ctx, cu = ints([common] * 3), cu_of(own)
    q = enter(sum(own), full, ctx, cu)
    out, lse = qf.attn_prefill(q, kc, vc, dev(full), dev(ctx), dev(cu))
    check_attention(out, lse, oracle.prefill(f64(q), f64(kc), f64(vc), full.numpy(), ctx.numpy(), cu.numpy(),
                                             SCALE))
    lens = ints([common + n for n in own])
    tail = full[:, whole:].contiguous()
    for _ in range(steps):
        q = enter(3, full, lens, None)
        lens = lens + 1
        out, lse = qf.attn_decode_shared(q, kc, vc, dev(one), dev(ints([16 * whole])), dev(ints([0, 3])),
                                         dev(tail), dev(lens - 16 * whole), 2, scale=SCALE)
        ref = oracle.decode_shared(f64(q), f64(kc), f64(vc), one.numpy(), [0], [0, 3], full.numpy(),
                                   lens.numpy(), SCALE)
        check_attention(out, lse, ref)


def _three_plans():
    a = rope_case(61, 8, 2, [40, 3], [9, 500], fused=True)
    p = prefill_case(62, 8, 2, [40, 3], [9, 1500])
    s = shared_case(63, 8, 2, [0, 3], [1200], [16, 0, 45, 7])
    d = lambda c, *names: [c[n].to(DEV) for n in names]  # noqa: E731
    plans = [qf.RopeAppendPlan(*d(a, "q", "k", "v", "kc", "vc", "table", "ctx", "cu"),
                               freqs=a["freqs"].to(DEV), q_gain=a["gains"][0].to(DEV),
                               k_gain=a["gains"][1].to(DEV)),
             qf.PrefillPlan(*d(p, "q", "kc", "vc", "table", "ctx", "cu")),
             qf.SharedDecodePlan(*d(s, "q", "kc", "vc", "pt", "pl", "rows", "table", "ctx", "ns"),
                                 max_shards=2)]
    return plans


def _results(plans):
    return [plans[0].q_out, plans[0]._keep[5], plans[0]._keep[6], plans[1].out, plans[1].lse,
            plans[2].out, plans[2].lse]


def test_streams_and_graphs(gpu):
    """On a side stream, captured in one graph and replayed several times with eager work and
    synchronisations between the replays: the bits of the eager calls every time."""
    eager = _three_plans()
    for p in eager:
        p()
    torch.cuda.synchronize()
    want = [x.clone() for x in _results(eager)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plans = _three_plans()
        for p in plans:
            p()
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(_results(plans), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = _three_plans_on_current(plans)
    for i in range(4):
        for x in _results(captured)[-4:]:
            x.fill_(float("nan"))
        captured[0].q_out.zero_()
        for p in eager:
            p()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(_results(captured), want)), i


def _three_plans_on_current(plans):
    """The same buffers as ``plans``, bound to the capturing stream."""
    import ctypes
    stream = torch.cuda.current_stream().cuda_stream
    for p in plans:
        p._args = p._args[:-1] + (ctypes.c_void_p(stream),)
        p()
    return plans


def test_two_prefills_at_once(gpu):
    """Two calls on two streams with workspaces of their own, key ranges included."""
    cases = [prefill_case(70 + i, 8, 2, [30, 3], [9, 3000], sharp=2.0) for i in range(2)]
    want = [run_prefill(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    plans = []
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            d = {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in c.items()}
            plans.append(qf.PrefillPlan(d["q"], d["kc"], d["vc"], d["table"], d["ctx"], d["cu"], scale=SCALE))
    torch.cuda.synchronize()
    for _ in range(5):
        for p in plans:
            p()
    torch.cuda.synchronize()
    for p, (o, l) in zip(plans, want):
        assert torch.equal(p.out, o) and torch.equal(p.lse, l)


def test_repeated_calls_give_the_same_bits(gpu):
    plans = _three_plans()
    first = None
    for _ in range(3):
        for p in plans:
            p()
        torch.cuda.synchronize()
        now = [x.clone() for x in _results(plans)]
        assert first is None or all(torch.equal(x, y) for x, y in zip(first, now))
        first = now
