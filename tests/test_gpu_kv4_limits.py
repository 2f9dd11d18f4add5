"""The 4-bit key/value cache at the ends of its ranges: values near and past fp16's largest."""
import numpy as np
import pytest
import torch

import kv4_plain as plain
import paper_2412_07174_amd as scap
from test_gpu_kv4 import BF, F, Cache, i32

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ values that fp16 has not
def top_is_a_number(s, c):
    """Whether what code 15 stands for is a number of fp16: 79 s + c is exact in fp64 (18 bits of a product and 11 more, not 2^15 apart
    where it matters), so the conversion is the one rounding."""
    with np.errstate(all="ignore"):
        return np.isfinite((79 * s.astype(np.float64) + c.astype(np.float64)).astype(np.float16)).all(-1)


def token_codes(k, v):
    """plain.token_codes with the last condition."""
    qk, sk, ck, a = plain.quantise(k)
    qv, sv, cv, b = plain.quantise(v)
    bad = ~(a & b & top_is_a_number(sk, ck) & top_is_a_number(sv, cv))
    for q in (qk, qv):
        q[bad] = 0
    for s in (sk, ck, sv, cv):
        s.view(np.uint16)[bad] = 0x7E00
    return qk, sk, ck, qv, sv, cv


# ends of a group; what is readable of it is token_codes' to say
ENDS = {BF: [(60000, 66000), (90000, 105000), (70400, 86900), (64000, 65000), (65280, 65280), (-105000, -90000), (-65280, -64000), (0, 15000),
             (-7000, 65280)],
        F: [(63648, 65504), (50144, 65504), (65504, 65504), (60000, 60100), (65440, 65504), (-65504, -63648), (-65504, -65504), (0, 15350)]}


def near_the_end(dt, n, heads, D, seed):
    """Tokens [n, heads, D] whose first group lies between ends such as these, or anywhere near them; the others are ordinary."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, heads, D), generator=g)
    t = torch.rand((n, heads, 32), generator=g)
    t[..., 0], t[..., 1] = 0, 1
    for i in range(n):
        for h in range(heads):
            if i < len(ENDS[dt]):
                lo, hi = ENDS[dt][i]
            else:
                hi = 65504 - 60 * float(torch.rand((), generator=g)) if dt == F else 40000 + 70000 * float(torch.rand((), generator=g))
                lo = hi - 16000 * float(torch.rand((), generator=g)) ** 2
            x[i, h, :32] = lo + t[i, h] * (hi - lo)
    return x.to(dt)


@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("D,P,n", [(64, 16, 300), (128, 64, 300), (128, 32, 2100)])
def test_append_of_values_that_fp16_has_not(dt, D, P, n, monkeypatch):
    """Bit for bit: unreadable where code 15 stands for no number of fp16, as before otherwise."""
    heads = 2
    c = Cache([n], heads, D, P, dt, seed=D)
    c.k[0][:300], c.v[0][-300:] = near_the_end(dt, 300, heads, D, 1), near_the_end(dt, 300, heads, D, 2)
    c.fill_all()
    monkeypatch.setattr(plain, "token_codes", token_codes)
    want = plain.Pool(c.pages, heads, D, P)
    for pos in range(n):
        want.put(c.table[0, pos // P], pos % P, c.k[0][pos].float().numpy(), c.v[0][pos].float().numpy())
    assert np.array_equal(c.cache.pool[0].cpu().numpy(), want.bytes)
    held = np.isfinite(c.stood_for(0)[0]).all(-1)
    assert 2 < (~held).sum() < 2 * n - 10, "both kinds occur"


@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_gives_what_the_cache_holds_near_the_end_of_fp16(dt, D, monkeypatch):
    """Sequences of one token, whose probability is 1: its value, rounded to fp16 by the widening and to the output's type, bit for bit;
    NaN where it cannot be read."""
    n, heads = 400, 2
    c = Cache([1] * n, heads, D, 16, dt, seed=5)
    x = near_the_end(dt, n, heads, D, 3)
    for b in range(n):
        c.v[b] = x[b:b + 1]
    c.fill_all()
    monkeypatch.setattr(plain, "token_codes", token_codes)
    ws = scap.KV4Workspace(c.cache, seqs=n, tokens=n, heads=4, max_new=1)
    q = torch.zeros((n, 4, D), dtype=dt, device="cuda")
    got = scap.kv4_attention(c.cache, q, i32(range(n + 1)), c.d_table, c.d_lens, max_new=1, workspace=ws).cpu()
    want = np.stack([c.stood_for(b)[1][0] for b in range(n)]).repeat(2, 1)
    unreadable = np.isnan(want)
    assert 2 < unreadable.any((1, 2)).sum() < n - 10, "both kinds occur"
    want = torch.from_numpy(want.astype(np.float16)).to(dt)
    assert np.array_equal(got.isnan().numpy(), unreadable) and torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))


@pytest.mark.parametrize("dt,lo,hi", [(BF, 70400, 86900), (BF, 60000, 66000), (F, 63648, 65504)])
@pytest.mark.parametrize("n,heads,window", [(5, 8, 0), (5, 8, 2), (70, 8, 0), (70, 8, 3), (280, 128, 0), (280, 128, 2)])
@pytest.mark.parametrize("where", ["k", "v"])
def test_a_finite_token_past_fp16_reaches_only_who_sees_it(dt, lo, hi, n, heads, window, where):
    """At the edge of what rows see: those before it, and those whose window has passed it, get the bits they get without it."""
    outs = []
    for large in (False, True):
        c = Cache([300, 90], 2, 128, 64, dt, seed=8)
        bad = 300 - n + 3
        if large:
            (c.k if where == "k" else c.v)[0][bad, 1, 32:64] = torch.linspace(lo, hi, 32).to(dt)
        c.fill_all()
        q = torch.randn((n + 1, heads, 128), generator=torch.Generator().manual_seed(1)).to(dt).cuda()
        ws = scap.KV4Workspace(c.cache, seqs=2, tokens=n + 1, heads=heads)
        outs.append(scap.kv4_attention(c.cache, q, i32([0, n, n + 1]), c.d_table, c.d_lens, window=window, workspace=ws).cpu())
    sees = torch.zeros((n + 1, heads), dtype=torch.bool)
    sees[3:min(3 + window, n) if window else n, heads // 2:] = True   # the upper half of the heads reads kv head 1
    assert bool(outs[1][sees].isnan().all())
    assert torch.equal(outs[1][~sees], outs[0][~sees]) and not bool(outs[0].isnan().any())


# ------------------------------------------------------------------------------------------------ pages
def test_a_fork_refuses_arrays_that_it_reads_and_takes_their_neighbours():
    cache = scap.KV4Cache(8, 1, 64, page_tokens=16)
    ints = i32(range(64))
    table, lens, parents, kids, kid_lens = ints[:6].view(2, 3), ints[6:8], ints[8:11], ints[11:20].view(3, 3), ints[20:23]
    table.copy_(i32([[5, 6, 7], [2, -1, -1]]))
    lens.copy_(i32([40, 3]))
    parents.copy_(i32([1, 0, 1]))
    before = ints.cpu()
    for out in (lens.view(-1), parents):
        n = out.shape[0]
        with pytest.raises(ValueError):
            scap.kv4_fork(cache, table, lens, parents[:n], kids[:n], out)
    with pytest.raises(ValueError):
        scap.kv4_fork(cache, table, lens, parents, ints[3:12].view(3, 3), kid_lens)
    assert torch.equal(ints.cpu(), before) and int(cache.refs.sum()) == 0
    scap.kv4_fork(cache, table, lens, parents, kids, kid_lens)   # side by side is apart
    assert kid_lens.tolist() == [3, 40, 3] and kids.tolist() == [[2, -1, -1], [5, 6, 7], [2, -1, -1]]
    assert cache.refs.tolist() == [0, 0, 2, 0, 0, 1, 1, 1]


@pytest.mark.parametrize("keep_from,keep_to", [([0, 1, 16, 17], None), ([40, 63, 64, 200], None), ([-5, 0, 48, 47], None),
                                               (None, [0, 1, 16, 17]), (None, [40, 63, 64, 200]), (None, [-3, 0, 1000, 33])])
def test_free_with_one_bound_keeps_what_lies_on_its_side(keep_from, keep_to):
    P, S = 16, 4
    cache = scap.KV4Cache(16, 1, 64, page_tokens=P)
    rows = np.arange(16, dtype=np.int32).reshape(4, S)
    table = i32(rows)
    cache.refs.fill_(1)
    scap.kv4_free(cache, table, **{k: i32(v) for k, v in (("keep_from", keep_from), ("keep_to", keep_to)) if v is not None})
    first, end = keep_from or [0] * 4, keep_to or [S * P] * 4
    kept = np.array([[bool(set(range(s * P, (s + 1) * P)) & set(range(first[b], end[b]))) for s in range(S)] for b in range(4)])
    assert np.array_equal(table.cpu().numpy(), np.where(kept, rows, -1))
    assert np.array_equal(cache.refs.cpu().numpy().reshape(4, S), kept.astype(np.int32))


# ------------------------------------------------------------------------------------------------ queries
@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("D,n,heads", [(64, 1, 4), (128, 5, 8), (128, 70, 8), (128, 280, 128), (64, 200, 64)])
@pytest.mark.parametrize("x", [float("inf"), float("-inf"), float("nan")])
def test_a_query_that_is_no_number_gives_none(dt, D, n, heads, x):
    """Whatever the signs of what it meets: an infinite score less the maximum is none either.  Other rows get the bits they get without it,
    and one that sees nothing is empty all the same."""
    c = Cache([300, 90], 2, D, 64, dt, seed=8)
    c.k[0][:, 0, 5] = c.k[0][:, 0, 5].abs() + 0.5     # x times this has one sign for the first half of the heads
    c.k[0][:, 0, 6] = -c.k[0][:, 0, 6].abs() - 0.5
    c.fill_all()
    starts = i32([0, n, n + 2])
    ws = scap.KV4Workspace(c.cache, seqs=2, tokens=n + 2, heads=heads)
    q = torch.randn((n + 2, heads, D), generator=torch.Generator().manual_seed(1)).to(dt).cuda()
    c.d_table[1] = -1                                 # the second sequence's pages are missing
    outs = []
    bad = torch.zeros((n + 2, heads), dtype=torch.bool)
    for put in (False, True):
        if put:
            for t in (0, n // 2, n):
                for h in (0, heads // 2 - 1, heads // 2):
                    q[t, h, 5 + t % 2] = x
                    bad[t, h] = t < n
        lse = torch.empty((n + 2, heads), device="cuda")
        outs.append((scap.kv4_attention(c.cache, q, starts, c.d_table, c.d_lens, lse=lse, workspace=ws).cpu(), lse.cpu()))
    (want, want_lse), (got, got_lse) = outs
    assert bool(got[bad].isnan().all()) and bool(got_lse[bad].isnan().all())
    assert torch.equal(got[~bad], want[~bad]) and torch.equal(got_lse[~bad], want_lse[~bad])
    assert bool((got[n:] == 0).all()) and not bool(want.isnan().any())


@pytest.mark.parametrize("D,n,heads,length", [(128, 1, 4, 1), (64, 1, 4, 300), (128, 5, 8, 300), (128, 70, 8, 300), (128, 280, 128, 300), (64, 200, 64, 300),
                                              (128, 1, 8, 9000)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("exponent,scale", [(3, 0.1), (18, 0.1), (19, 0.1), (21, 0.1), (25, 0.1), (40, 0.1), (90, 0.1), (118, 0.1), (0, 1e9), (-60, 1e30)])
def test_scores_of_any_size(D, n, heads, length, sign, exponent, scale):
    """One key is far the best of every row, by more than any rounding: the output is its value's, bit for bit, however large the scores
    are, of either sign; their logarithm is the best one's."""
    best = 7 if length > 7 else 0
    c = Cache([length], 2, D, 64, BF, seed=9)
    pattern = torch.randint(0, 2, (D,), generator=torch.Generator().manual_seed(2)) * 2.0 - 1
    size = 1.5 + torch.rand((length, 2, 1), generator=torch.Generator().manual_seed(3))
    size[best] = 4.0 if sign > 0 else 0.75
    c.k[0] = (size * pattern).to(BF)
    c.fill_all()
    q = (sign * 2.0 ** exponent * pattern).to(BF).expand(n, heads, D).contiguous().cuda()
    ws = scap.KV4Workspace(c.cache, seqs=1, tokens=n, heads=heads)
    lse = torch.empty((n, heads), device="cuda")
    got = scap.kv4_attention(c.cache, q, i32([0, n]), c.d_table, c.d_lens, scale=scale, lse=lse, workspace=ws).cpu()
    k, v = c.stood_for(0)
    want = torch.from_numpy(v[best].astype(np.float16)).to(BF).repeat_interleave(heads // 2, 0)
    assert torch.equal(got, want.expand_as(got)), (got.float() - want.float()).abs().max()
    z = scale * sign * 2.0 ** exponent * (k @ pattern.double().numpy())     # [length, 2]
    top = np.sort(z, 0)[::-1]
    assert length == 1 or (top[0] - top[1] > 25).all(), "exp(-25) of length values moves no bit of them"
    want_lse = torch.from_numpy(z[best]).repeat_interleave(heads // 2)
    # keys carry 2^-11 each, the scale and its logarithm's base 2^-24 each
    assert bool(((lse.cpu().double() - want_lse).abs() <= 1.01 * 2.0 ** -11 * want_lse.abs() + 1e-4).all())


@pytest.mark.parametrize("old,new", [(50, 130), (50, 97), (48, 200), (0, 256), (3, 4), (130, 131), (50, 50)])
def test_a_row_cut_before_what_its_window_kept_loses_no_page(old, new):
    """refs stays the number of entries that name a page, whatever gap lies between the new end and what is left behind it."""
    P, S = 16, 16
    cache = scap.KV4Cache(40, 1, 64, page_tokens=P)
    ws = scap.KV4Workspace(cache, seqs=2)
    table = torch.full((2, S), -1, dtype=torch.int32, device="cuda")
    assert scap.kv4_reserve(cache, table, i32([0, 0]), i32([200, 30]), workspace=ws).tolist() == [0, 15, 0, 25]
    scap.kv4_free(cache, table, keep_from=i32([100, 0]))
    kept = table[0].clone()
    assert kept.tolist()[:6] == [-1] * 6 and kept[6:13].min() >= 0
    info = scap.kv4_reserve(cache, table, i32([old, 30]), i32([new, 30]), workspace=ws).tolist()
    rows = table.cpu().numpy()
    assert np.array_equal(np.bincount(rows[rows >= 0], minlength=40), cache.refs.cpu().numpy())
    assert info[0] == 0 and info[3] == int((cache.refs == 0).sum())
    if new > old:   # every slot that the new tokens take has a page of its own
        mine = rows[0, old // P:-(-new // P)]
        assert (mine >= 0).all() and len(set(rows[rows >= 0].tolist())) == (rows >= 0).sum()


def test_the_drop_of_a_long_cut_end():
    """More pages behind the old length than are looked at together, up to the row's end."""
    for S in (1, 2, 3, 4, 5, 7, 8, 9, 33):
        cache = scap.KV4Cache(S + 1, 1, 64, page_tokens=16)
        ws = scap.KV4Workspace(cache, seqs=1)
        for keep in range(0, S + 1, 3):
            cache.refs.zero_()
            table = torch.full((1, S), -1, dtype=torch.int32, device="cuda")
            scap.kv4_reserve(cache, table, i32([0]), i32([16 * S]), workspace=ws)
            before = table.clone()
            assert scap.kv4_reserve(cache, table, i32([16 * keep]), i32([16 * keep]), workspace=ws).tolist() == [0, 0, 0, S + 1 - keep]
            assert torch.equal(table[:, :keep], before[:, :keep]) and bool((table[:, keep:] == -1).all()) and int(cache.refs.sum()) == keep


# ------------------------------------------------------------------------------------------------ the quantiser's roundings
def tied(dt, n, heads, groups, seed):
    """Groups [n, heads, groups * 32] whose range is 15 times a number that lies midway between two of fp16, exactly: their quotient in fp32 is the
    tie itself, and any other way to round it to fp16 tells."""
    rng = np.random.default_rng(seed)
    shape = (n, heads, groups)
    e = rng.integers(-25 if dt == BF else -24, -4, shape)
    t = 2 * rng.integers(1024, 2048, shape) + 1                      # 12 bits, the last one set
    if dt == BF:
        small = e == -25                                             # below fp16's normal range fewer bits make a tie
        t = np.where(small, 2 * rng.integers(0, 1024, shape) + 1, t)
    r = 15 * t
    keep = 8 if dt == BF else 11
    drop = np.maximum(np.floor(np.log2(r)).astype(np.int64) + 1 - keep, 0)
    hi = r >> drop << drop
    lo = hi - r                                                      # as many bits as the kind has, or fewer
    x = lo[..., None] + rng.random(shape + (32,)) * r[..., None]
    x[..., 5], x[..., 17] = lo, hi
    x = torch.from_numpy(np.ldexp(x, e[..., None]).astype(np.float32)).to(dt).float()
    scaled = lambda a: torch.from_numpy(np.ldexp(a.astype(np.float64), e).astype(np.float32))[..., None]
    x = torch.minimum(torch.maximum(x, scaled(lo)), scaled(hi))
    assert torch.equal(x.to(dt).float(), x)
    return x.reshape(n, heads, groups * 32).to(dt)


def scattered(dt, n, heads, groups, seed):
    """Groups of any size, some far from zero, some with members of very different size."""
    rng = np.random.default_rng(seed)
    size = np.exp2(rng.uniform(-26, 9, (n, heads, groups, 1)))
    x = rng.standard_normal((n, heads, groups, 32)) * size
    x += np.where(rng.random((n, heads, groups, 1)) < 0.3, size * rng.uniform(-60, 60, (n, heads, groups, 1)), 0)
    x *= np.where(rng.random((n, heads, groups, 1)) < 0.3, np.exp2(rng.uniform(-20, 0, x.shape)), 1)
    return torch.from_numpy(x.reshape(n, heads, groups * 32).astype(np.float32)).to(dt)


@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("D,n", [(64, 1000), (128, 4032)])
@pytest.mark.parametrize("make", [tied, scattered])
def test_append_rounds_as_defined(dt, D, n, make):
    """Scales and codes of many groups, bit for bit."""
    P, heads = 64, 4
    pages = -(-n // P)
    k, v = make(dt, n, heads, D // 32, 1), make(dt, n, heads, D // 32, 2)
    cache = scap.KV4Cache(pages, heads, D, page_tokens=P)
    cache.pool.zero_()
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None].contiguous()
    scap.kv4_append(cache, k.cuda(), v.cuda(), i32([0, n]), table, i32([n]))
    pool = cache.pool[0].cpu().numpy()
    tokens = lambda a: a.transpose(0, 2, 1, *range(3, a.ndim)).reshape(pages * P, heads, -1)[:n]
    kc = pool[:, :, :P * D // 2].reshape(pages, heads, P, D // 2)
    vc = pool[:, :, P * D // 2:P * D].reshape(pages, heads, P // 4, D // 8, 4, 4).transpose(0, 1, 2, 4, 3, 5).reshape(pages, heads, P, D // 2)
    ks = np.ascontiguousarray(pool[:, :, P * D:P * D * 9 // 8]).view(np.uint16).reshape(pages, heads, P, D // 32, 2)
    vs = np.ascontiguousarray(pool[:, :, P * D * 9 // 8:]).view(np.uint16).reshape(pages, heads, P // 4, D // 32, 2, 4)
    vs = vs.transpose(0, 1, 2, 5, 3, 4).reshape(pages, heads, P, D // 32, 2)
    qk, sk, ck, qv, sv, cv = token_codes(k.float().numpy(), v.float().numpy())
    for codes, scales, q, s, c, x in ((kc, ks, qk, sk, ck, k), (vc, vs, qv, sv, cv, v)):
        # -0 counts as less than 0, which numpy's minimum does not tell; c is the least member where s is 0
        g = x.float().reshape(n, heads, D // 32, 32).numpy()
        least = np.where(((g == 0) & np.signbit(g)).any(-1), np.float16(-0.0), np.float16(0.0))
        c = np.where((s == 0) & (g.min(-1) == 0), least, c)
        assert np.array_equal(tokens(scales[..., 0]), s.view(np.uint16)), "s"
        assert np.array_equal(tokens(scales[..., 1]), c.view(np.uint16)), "c"
        codes = tokens(codes)
        assert np.array_equal(codes & 15, q[..., 0::2]) and np.array_equal(codes >> 4, q[..., 1::2]), "codes"


@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("D,n", [(64, 1), (128, 40)])
def test_values_and_scales_below_fp16s_normal_range(dt, D, n):
    """Nothing is flushed: one token's value of that size comes back as its fp16 number, whose place in the output's type it has."""
    seqs, heads = 60, 2
    c = Cache([1] * seqs, heads, D, 16, dt, seed=5)
    size = torch.exp2(-torch.linspace(10, 24, seqs))
    for b in range(seqs):
        c.v[b] = (c.v[b].float() * size[b]).to(dt)
        c.k[b] = (c.k[b].float() * size[b]).to(dt)
    c.fill_all()
    news = [n] * seqs                                   # the last of a sequence's new tokens sees its one token
    ws = scap.KV4Workspace(c.cache, seqs=seqs, tokens=n * seqs, heads=2 * heads)
    q = torch.randn((n * seqs, 2 * heads, D), generator=torch.Generator().manual_seed(3)).to(dt).cuda()
    out = scap.kv4_attention(c.cache, q, i32(np.cumsum([0] + news)), c.d_table, c.d_lens, workspace=ws)[n - 1::n].cpu()
    want = np.stack([c.stood_for(b)[1][0] for b in range(seqs)]).repeat(2, 1)
    assert torch.equal(out, torch.from_numpy(want.astype(np.float16)).to(dt)) and bool((out != 0).any(-1).all())
