"""Operators around paged caches against their definitions in 64 bits.

Tolerances are derived from the arithmetic: u = 2^-24 is half a step of fp32 at 1, an output rounded to type t is off by at most
finfo(t).eps / 2 of its value, and a score is a sum of head_dim products of fp32 numbers."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": U, "bf16": 2.0 ** -8}


def rt_module():
    from paper_2604_21215_b200 import rt
    return rt


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def make_cache(lens, kv, hd, page, cache, seed=0, spare=3, slack=1, nan_behind=True):
    """A cache whose sequences hold random pairs; its page numbers are shuffled, places behind the lengths and pages that nobody owns hold
    NaN, and table entries behind a sequence's pages name pages that do not exist.  -> PagedCache, k, v in 64 bits [b][n, kv, hd]"""
    rt = rt_module()
    g = gen(seed)
    need = [-(-max(n, 0) // page) for n in lens]
    n_pages = sum(need) + spare
    c = rt.PagedCache.empty(n_pages, page, kv, len(lens), max(max(need), 1) + slack, head_dim=hd, dtype=cache)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).int()
    table = torch.full(tuple(c.page_table.shape), 1 << 30, dtype=torch.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    c.page_table.copy_(table)
    if nan_behind:
        for pool in (c.k, c.v):
            pool.view(torch.uint8 if cache == "e4m3" else pool.dtype).fill_(0x7f if cache == "e4m3" else math.nan)
    seq = torch.tensor([b for b, n in enumerate(lens) for _ in range(n)], dtype=torch.int32, device="cuda")
    pos = torch.tensor([i for n in lens for i in range(n)], dtype=torch.int32, device="cuda")
    k = torch.randn((len(seq), kv, hd), generator=g, device="cuda")
    v = torch.randn((len(seq), kv, hd), generator=g, device="cuda") * torch.exp(torch.randn((len(seq), kv, 1), generator=g, device="cuda"))
    if cache == "bf16":
        k, v = k.bfloat16(), v.bfloat16()
    c.write(k, v, seq, pos)
    k, v = c.read(seq, pos, dtype="f32")                       # what the cache stands for (exact in fp32)
    cut = [max(n, 0) for n in lens]
    return c, k.double().split(cut), v.double().split(cut)


def reference(q, ks, vs, lens, k_own=None, v_own=None, scale=None, slopes=None):
    """out, lse in 64 bits, and the bounds of an fp32 evaluation's error (before the rounding of out)."""
    B, H, hd = q.shape
    outs, lses, eo, el = [], [], [], []
    q = q.double()
    for b in range(B):
        k, v = ks[b], vs[b]
        n = len(k)
        dist = (n if k_own is not None else n - 1) - torch.arange(n, device="cuda", dtype=torch.float64)
        if k_own is not None:
            k, v = torch.cat((k, k_own[b:b + 1].double())), torch.cat((v, v_own[b:b + 1].double()))
            dist = torch.cat((dist, dist.new_zeros(1)))
        group = H // k.shape[1]
        k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
        s = 1.0 / math.sqrt(hd) if scale is None else scale
        a = torch.einsum("hd,nhd->hn", q[b], k) * s
        size = torch.einsum("hd,nhd->hn", q[b].abs(), k.abs()) * abs(s)
        if slopes is not None:
            a = a - slopes.double()[:, None] * dist
            size = size + slopes.double().abs()[:, None] * dist.abs()
        if not len(k):
            outs.append(q.new_zeros(H, hd)); lses.append(q.new_full((H,), -math.inf)); eo.append(q.new_zeros(H, hd)); el.append(q.new_zeros(H))
            continue
        p = torch.softmax(a, 1)
        o = torch.einsum("hn,nhd->hd", p, v)
        # a score's error: hd products and sums, the factors of scale and of log2(e); a weight's: that of its score and of exp2, twice (weight and
        # sum), and sums of len(k) terms; all relative to sum_j p_j |v_j|
        ea = (p * size).sum(1) * (hd + 8) * U
        rel = 2 * ea + (len(k) + 40) * U + 2.0 ** -20
        outs.append(o); lses.append(torch.logsumexp(a, 1))
        eo.append(rel[:, None] * torch.einsum("hn,nhd->hd", p, v.abs()) + 2 * ((p * size)[:, :, None] * (v.transpose(0, 1) - o[:, None]).abs()).sum(1) * (hd + 8) * U)
        el.append(ea + (len(k) + 40) * U + 4 * U * lses[-1].abs() + 2.0 ** -20)
    return torch.stack(outs), torch.stack(lses), torch.stack(eo), torch.stack(el)


def check(out, lse, ref, dtype):
    o, l, eo, el = ref
    assert torch.isfinite(out.float()).all()
    bound = HALF_STEP[dtype] * (o.abs() + eo) + eo + 1e-30
    worst = ((out.double() - o).abs() / bound).max().item()
    assert worst <= 1.0, worst
    if lse is not None:
        empty = torch.isinf(l)
        assert torch.equal(torch.isinf(lse), empty)
        assert ((lse.double() - l).abs() <= el)[~empty].all()


SHAPES = [  # lens, heads, kv, hd, page
    ([1], 1, 1, 64, 16),
    ([0, 1, 2, 15, 16, 17, 31, 33], 2, 2, 64, 16),
    ([257, 0, 1000, 64, 65], 12, 12, 64, 16),
    ([100, 3, 511], 8, 2, 64, 32),
    ([129, 128, 127, 1], 6, 2, 64, 64),
    ([5, 700], 8, 1, 64, 128),
    ([255, 256, 257, 513], 5, 5, 128, 256),
    ([300, 77], 16, 2, 128, 16),
    ([40, 1025], 10, 2, 64, 16),
    ([333], 24, 1, 128, 32),
    ([90, 2000], 17, 1, 64, 16),
    ([4097], 3, 3, 64, 16),
]


@pytest.mark.parametrize("room", ["little", "much"])                    # positions that the page table could hold
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("f32", "e4m3"), ("f32", "bf16"), ("bf16", "f32")])
def test_attention_of_one_token(shape, dtype, cache, room):
    lens, H, kv, hd, page = shape
    c, ks, vs = make_cache(lens, kv, hd, page, cache, seed=len(lens) * hd + H, slack=1 if room == "little" else 40000 // page)
    g = gen(5)
    t, B = TYPES[dtype], len(lens)
    q = torch.randn((B, H, hd), generator=g, device="cuda").to(t)
    ko, vo = (torch.randn((B, kv, hd), generator=g, device="cuda").to(t) for _ in range(2))
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device="cuda")
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for own in (False, True):
        for sl in (None, slopes):
            lse = torch.full((B, H), 7.0, device="cuda")
            kw = dict(k_own=ko, v_own=vo) if own else {}
            out = c.attend(q, n, alibi_slopes=sl, lse=lse, **kw)
            check(out, lse, reference(q, ks, vs, lens, ko if own else None, vo if own else None, None, sl), dtype)
            if own is False:
                for b in [i for i, x in enumerate(lens) if x == 0]:        # nothing to attend to
                    assert (out[b] == 0).all() and (lse[b] == -math.inf).all()
    torch.cuda.synchronize()
    assert c.status() == 0


@pytest.mark.parametrize("n_seqs,H,kv,cache", [(300, 2, 2, "bf16"), (700, 4, 2, "e4m3"), (1500, 1, 1, "f32")])
def test_attention_of_large_ragged_batches(n_seqs, H, kv, cache):
    # several sequences for each thread that adds up the lengths, more heads than the join has blocks, empty and unused rows in between
    rng = np.random.default_rng(n_seqs)
    lens = [int(x) for x in rng.choice([-1, 0, 1, 16, 33, 50, 100, 400], n_seqs, p=[0.1, 0.1, 0.1, 0.1, 0.2, 0.2, 0.15, 0.05])]
    c, ks, vs = make_cache([max(x, 0) for x in lens], kv, 64, 16, cache, seed=n_seqs)
    q = torch.randn((n_seqs, H, 64), generator=gen(1), device="cuda")
    ko, vo = (torch.randn((n_seqs, kv, 64), generator=gen(s), device="cuda") for s in (2, 3))
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = torch.full((n_seqs, H, 64), 4.0, device="cuda"), torch.full((n_seqs, H), 4.0, device="cuda")
    c.attend(q, n, k_own=ko, v_own=vo, out=out, lse=lse)
    used = n >= 0
    assert (out[~used] == 4.0).all() and (lse[~used] == 4.0).all()
    ref = reference(q, ks, vs, lens, ko, vo)
    check(out[used], lse[used], tuple(x[used] for x in ref), "f32")


@pytest.mark.parametrize("cache,lens", [("bf16", [20011]), ("f32", [20011]), ("e4m3", [60001]), ("bf16", [3, 30000, 1, 7])])
def test_attention_of_one_long_sequence(cache, lens):
    # one head shared by hundreds of warps
    c, ks, vs = make_cache(lens, 1, 64, 64, cache, seed=4)
    q = torch.randn((len(lens), 2, 64), generator=gen(1), device="cuda")
    lse = torch.empty((len(lens), 2), device="cuda")
    slopes = torch.tensor([2.0 ** -8, 2.0 ** -12], device="cuda")
    for sl in (None, slopes):
        out = c.attend(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), alibi_slopes=sl, lse=lse)
        check(out, lse, reference(q, ks, vs, lens, slopes=sl), "f32")


@pytest.mark.parametrize("slack", [1, 4000])
def test_attention_with_sharp_and_flat_scores(slack):
    # one key far above the others early or late in the sequence (the running maximum moves), all scores equal, a scale of zero
    lens, H, hd = [700, 700, 300], 2, 64
    c, ks, vs = make_cache(lens, H, hd, 16, "f32", seed=3, slack=slack)
    q = torch.randn((3, H, hd), generator=gen(1), device="cuda")
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    seq, pos = torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.tensor([2, 690], dtype=torch.int32, device="cuda")
    k = torch.stack((q[0], q[1])) * 4
    v = torch.randn((2, H, hd), generator=gen(2), device="cuda")
    c.write(k, v, seq, pos)
    for b, j in ((0, 2), (1, 690)):
        ks[b][j], vs[b][j] = k[b].double(), v[b].double()
    for scale in (None, 0.0, 1.0, -0.5):
        lse = torch.empty((3, H), device="cuda")
        check(c.attend(q, n, scale=scale, lse=lse), lse, reference(q, ks, vs, lens, scale=scale), "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("order", [1, -1])
def test_attention_over_rows_of_very_different_scales(dtype, order):
    # 8-bit pages whose rows span 2^-20 to 2^20, growing or shrinking along the sequence, weighted towards either end
    rt = rt_module()
    B, H, n = 3, 2, 500
    c = rt.PagedCache.empty(B * 32, 16, H, B, 32, dtype="e4m3")
    c.page_table.copy_(torch.arange(B * 32).view(B, 32).int())
    seq, pos = torch.arange(B, device="cuda").int().repeat_interleave(n), torch.arange(n, device="cuda").int().repeat(B)
    grow = 2.0 ** (order * (torch.arange(n, device="cuda", dtype=torch.float64) / n * 40 - 20)).float().repeat(B)[:, None, None]
    k = torch.randn((B * n, H, 64), generator=gen(1), device="cuda") * torch.exp2(torch.randint(-3, 2, (B * n, H, 1), generator=gen(5), device="cuda").float())
    v = torch.randn((B * n, H, 64), generator=gen(2), device="cuda") * grow
    c.write(k, v, seq, pos)
    k, v = (x.double().split([n] * B) for x in c.read(seq, pos, dtype="f32"))
    q = torch.randn((B, H, 64), generator=gen(3), device="cuda").to(TYPES[dtype])
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    for slopes in (None, torch.tensor([0.03, -0.03], device="cuda"), torch.tensor([0.2, 2.0], device="cuda")):
        lse = torch.empty((B, H), device="cuda")
        out = c.attend(q, lens, alibi_slopes=slopes, lse=lse)
        check(out, lse, reference(q, k, v, [n] * B, slopes=slopes), dtype)


@pytest.mark.parametrize("slack", [1, 4000])
def test_infinities_and_nan_count_where_they_are_attended_to(slack):
    # a NaN key or value shows in its own head and sequence only; an infinite value as itself; places that are not attended to never show
    for cache in ("f32", "bf16"):
        c, ks, vs = make_cache([40, 40, 40], 2, 64, 16, cache, seed=9, slack=slack)
        n = torch.tensor([40, 40, 39], dtype=torch.int32, device="cuda")
        place = lambda b, j: (int(c.page_table[b, j // 16]), j % 16)
        p, o = place(0, 20)
        c.k[p, 0, o, 5] = math.nan
        p, o = place(1, 20)
        c.v[p, 1, o, 7] = math.inf
        p, o = place(2, 39)
        c.k[p, :, o], c.v[p, :, o] = math.nan, math.inf
        q = torch.randn((3, 2, 64), generator=gen(4), device="cuda").to(TYPES[cache])
        out = c.attend(q, n).float()
        assert torch.isnan(out[0, 0]).all() and torch.isfinite(out[0, 1]).all()
        assert torch.isfinite(out[1, 0]).all() and out[1, 1, 7] == math.inf and torch.isfinite(out[1, 1, :7]).all()
        assert torch.isfinite(out[2]).all()


@pytest.mark.parametrize("slack", [1, 4000])
def test_rows_not_in_use_stay_and_strided_rows_are_taken(slack):
    lens, H, kv, hd = [33, -1, 50, -5], 4, 2, 64
    for cache in ("bf16", "f32"):
        t = TYPES[cache]
        c, ks, vs = make_cache([33, 0, 50, 0], kv, hd, 16, cache, seed=2, slack=slack)
        wide = torch.randn((4, (H + 2 * kv) * hd + 16), generator=gen(3), device="cuda").to(t)        # q | k | v | padding
        q, ko, vo = (wide[:, a * hd:b * hd].view(4, -1, hd) for a, b in ((0, H), (H, H + kv), (H + kv, H + 2 * kv)))
        big = torch.full((4, 2 * H * hd), 3.0, device="cuda", dtype=t)
        out, lse = big[:, H * hd:].view(4, H, hd), torch.full((4, H), 5.0, device="cuda")
        got = c.attend(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), k_own=ko, v_own=vo, out=out, lse=lse)
        assert got is out and (big[:, :H * hd] == 3.0).all()
        assert (out[[1, 3]] == 3.0).all() and (lse[[1, 3]] == 5.0).all()
        ref = reference(q, ks, vs, lens, ko, vo)
        keep = [0, 2]
        check(out[keep], lse[keep], tuple(x[keep] for x in ref), cache)


@pytest.mark.parametrize("cache,more", [("f32", 0), ("f32", 90), ("bf16", 0), ("bf16", 90)])
def test_pages_and_lengths_that_do_not_exist(cache, more):
    # (more: sequences behind these)
    rt = rt_module()
    lens = [70, 200, 64]
    c, ks, vs = make_cache(lens + [1] * more, 2, 64, 16, cache, seed=6, slack=0)
    run = lambda q, n, lse=None: c.attend(torch.cat((q, q[:1].expand(more, -1, -1))), torch.cat((n, torch.ones(more, dtype=torch.int32, device="cuda"))),
                                          lse=None if lse is None else big)[:3]
    big = torch.empty((3 + more, 2), device="cuda")
    q = torch.randn((3, 2, 64), generator=gen(4), device="cuda")
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    run(q, n)
    torch.cuda.synchronize()
    assert c.status() == rt.RT_OK
    ks, vs = ks[:3], vs[:3]
    for bad in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        old = int(c.page_table[1, 3])
        c.page_table[1, 3] = bad
        out = run(q, n, big)
        lse = big[:3]
        torch.cuda.synchronize()
        assert c.status() == rt.RT_ERR_INVALID_ARG
        c.page_table[1, 3] = old
        c.clear_status()
        cut = lambda x: [x[0], torch.cat((x[1][:48], x[1][64:])), x[2]]        # the pairs of that page have no weight
        check(out, lse, reference(q, cut(ks), cut(vs), lens), "f32")
    # a length beyond the table is cut to it
    long = torch.tensor([70, 2 ** 31 - 1, 64], dtype=torch.int32, device="cuda")
    full = c.page_table.shape[1] * 16
    assert full == 208
    pos = torch.arange(200, 208, dtype=torch.int32, device="cuda")
    kx = torch.randn((8, 2, 64), generator=gen(8), device="cuda").bfloat16().float()
    c.write(kx, kx, torch.ones_like(pos), pos)
    out = run(q, long)
    torch.cuda.synchronize()
    assert c.status() == rt.RT_ERR_INVALID_ARG
    ref = reference(q, [ks[0], torch.cat((ks[1], kx.double())), ks[2]], [vs[0], torch.cat((vs[1], kx.double())), vs[2]], lens)
    check(out, None, ref, "f32")


def test_writes_and_reads_of_places_that_do_not_exist():
    rt = rt_module()
    for cache in ("bf16", "e4m3"):
        c, ks, vs = make_cache([40, 20], 2, 64, 16, cache, seed=1, nan_behind=False)
        before = [x.clone() for x in (c.k.view(torch.uint8), c.v.view(torch.uint8)) + ((c.k_exp, c.v_exp) if cache == "e4m3" else ())]
        T = c.page_table.shape[1] * 16
        seq = torch.tensor([0, 2, -1, 0, 1, 0, 1], dtype=torch.int32, device="cuda")
        pos = torch.tensor([-1, 0, 3, T, 2 ** 31 - 1, -2 ** 31, 47], dtype=torch.int32, device="cuda")       # (the last: a table entry that names no page)
        x = torch.randn((7, 2, 64), generator=gen(2), device="cuda").bfloat16()
        c.write(x[:1], x[:1], seq[:1], pos[:1])
        torch.cuda.synchronize()
        assert c.status() == rt.RT_OK                          # a negative position is no error
        c.write(x, x, seq, pos)
        k, v = (torch.full((7, 2, 64), 9.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        c.read(seq, pos, k=k, v=v)
        torch.cuda.synchronize()
        assert c.status() == rt.RT_ERR_INVALID_ARG
        assert (k == 9.0).all() and (v == 9.0).all()
        after = (c.k.view(torch.uint8), c.v.view(torch.uint8)) + ((c.k_exp, c.v_exp) if cache == "e4m3" else ())
        assert all(torch.equal(a, b) for a, b in zip(before, after))


def quantised(x):
    """(codes, exponents) of rows, on the CPU: all steps but the rounding to e4m3 are exact."""
    x = x.cpu().float()
    fine = torch.isfinite(x)
    most = torch.where(fine, x.abs(), 0.0).amax(-1).double().numpy()
    m, e = np.frexp(most)
    k = np.where(most > 0, e - 9 + (m > 0.875), -126).clip(min=-126)
    y = np.ldexp(x.double().numpy(), -k[..., None].astype(np.int64))
    y = torch.from_numpy(np.where(fine.numpy(), y, np.nan))
    # to nearest, ties to even, on e4m3's grid of steps 2^(floor(log2 |y|) - 3), at least 2^-9
    step = 2.0 ** (torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, torch.from_numpy(k + 127)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd,page,kv", [(64, 16, 1), (64, 64, 3), (128, 32, 2)])
def test_rows_in_8_bits_are_the_nearest_codes(dtype, hd, page, kv):
    rt = rt_module()
    lens = [100, 1, 0, 37]
    g = gen(11)
    c = rt.PagedCache.empty(40, page, kv, 4, 16, head_dim=hd, dtype="e4m3")
    c.page_table.copy_(torch.randperm(64, generator=torch.Generator().manual_seed(1))[:64].view(4, 16).int() % 40)
    c.page_table[0, :7], c.page_table[1, 0], c.page_table[3, :3] = torch.arange(7).int(), 7, torch.arange(8, 11).int()
    seq = torch.tensor([b for b, n in enumerate(lens) for _ in range(n)], dtype=torch.int32, device="cuda")
    pos = torch.tensor([i for n in lens for i in range(n)], dtype=torch.int32, device="cuda")
    R = len(seq)
    order = torch.randperm(R, generator=torch.Generator().manual_seed(2)).cuda()       # rows in any order
    seq, pos = seq[order], pos[order]
    k = torch.randn((R, kv, hd), generator=g, device="cuda") * torch.exp(8 * torch.randn((R, kv, 1), generator=g, device="cuda"))
    v = torch.randn((R, kv, hd), generator=g, device="cuda")
    for i, x in enumerate((0.0, -0.0, 448.0, 449.0, 448.0 * 2.0 ** -126, 1e-40, 2.0 ** -149, 3.0e38, 3.4028234e38, math.inf, -math.inf, math.nan, 447.9, 1.75, 1.7500001, 224.0)):
        k[i, 0] = x                                                    # rows at the borders of the scale's choice
        v[i, 0, 1:] *= 1e-3
        v[i, 0, 0] = x
    v[20, 0] = torch.linspace(-448, 448, hd, device="cuda")
    v[21, 0, :16], v[21, 0, 16:] = 448.0, 2.0 ** -9 * torch.arange(hd - 16, device="cuda") / 2       # subnormal codes and ties between them
    k, v = k.to(TYPES[dtype]), v.to(TYPES[dtype])
    before = c.k.view(torch.uint8).clone()
    c.write(k, v, seq, pos)
    for x, pool, exps in ((k, c.k, c.k_exp), (v, c.v, c.v_exp)):
        want, e = quantised(x)
        page_no, off = c.page_table[seq.long(), pos.long() // page].long(), pos.long() % page
        got = pool.view(torch.uint8)[page_no, :, off].view(torch.float8_e4m3fn).double().cpu()
        assert torch.equal(exps[page_no, :, off].cpu().long(), e.long())
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))
    touched = torch.zeros((40, page), dtype=torch.bool, device="cuda")
    touched[page_no, off] = True
    assert torch.equal(c.k.view(torch.uint8).transpose(1, 2)[~touched], before.transpose(1, 2)[~touched])     # nothing else is written
    for out in ("f32", "bf16"):
        kr, vr = c.read(seq, pos, dtype=out)
        for r, x in ((kr, k), (vr, v)):
            want, e = quantised(x)
            want = want * 2.0 ** (e.double()[..., None] - 127)           # exact in both types, but for bf16's overflow and subnormals
            want = want.float().to(TYPES[out]).double()
            got = r.double().cpu()
            assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_rows_in_the_storage_types(dtype, cache):
    rt = rt_module()
    c = rt.PagedCache.empty(9, 16, 3, 2, 4, dtype=cache)
    c.page_table.copy_(torch.tensor([[8, 1, 7, 0], [3, 2, 6, 5]], dtype=torch.int32))
    seq = torch.tensor([0, 1, 0, 1, 1], dtype=torch.int32, device="cuda")
    pos = torch.tensor([63, 0, 16, 15, 33], dtype=torch.int32, device="cuda")
    qkv = torch.randn((5, 1000), generator=gen(1), device="cuda").to(TYPES[dtype])
    k, v = qkv[:, 8:200].view(5, 3, 64), qkv[:, 304:496].view(5, 3, 64)
    c.write(k, v, seq, pos)
    for x, pool in ((k, c.k), (v, c.v)):
        at = pool[c.page_table[seq.long(), pos.long() // 16].long(), :, pos.long() % 16]
        assert torch.equal(at, x.to(TYPES[cache]))
    assert (c.k == 0).all(3).sum() == 9 * 3 * 16 - 15
    kr, vr = c.read(seq, pos, dtype=dtype)
    assert torch.equal(kr, k.to(TYPES[cache]).to(TYPES[dtype])) and torch.equal(vr, v.to(TYPES[cache]).to(TYPES[dtype]))


@pytest.mark.parametrize("dtype,cache", [("f32", "e4m3"), ("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32")])
@pytest.mark.parametrize("rows,kv,hd", [(5003, 1, 64), (4000, 3, 64), (3001, 16, 64), (2500, 5, 128)])
def test_many_rows(rows, kv, hd, dtype, cache):
    # several rows a warp, some of them not in use, caches of few and of many heads
    rt = rt_module()
    B, page = 7, 32
    per = -(-rows // B)
    pages = -(-per // page)
    c = rt.PagedCache.empty(B * pages, page, kv, B, pages, head_dim=hd, dtype=cache)
    c.page_table.copy_(torch.randperm(B * pages, generator=torch.Generator().manual_seed(1)).view(B, pages).int())
    order = torch.randperm(B * per, generator=torch.Generator().manual_seed(2))[:rows].cuda()
    seq, pos = (order // per).int(), (order % per).int()
    k, v = (torch.randn((rows, kv, hd), generator=gen(s), device="cuda").to(TYPES[dtype]) for s in (1, 2))
    skip = torch.rand(rows, generator=gen(3), device="cuda") < 0.2
    c.write(k, v, seq, torch.where(skip, -1, pos))
    kr, vr = (torch.full((rows, kv, hd), 6.0, device="cuda") for _ in range(2))
    c.read(seq, torch.where(skip, -1, pos), dtype="f32", k=kr, v=vr)
    torch.cuda.synchronize()
    assert c.status() == 0
    for got, x in ((kr, k), (vr, v)):
        assert (got[skip] == 6.0).all()
        if cache == "e4m3":
            want, e = quantised(x[~skip])
            want = (want * 2.0 ** (e.double()[..., None] - 127)).float().cuda()
        else:
            want = x[~skip].to(TYPES[cache]).float()
        assert torch.equal(got[~skip], want)
    kr, vr = c.read(seq[skip], pos[skip], dtype="f32")                  # what was skipped is not there
    assert (kr == 0).all() and (vr == 0).all()


def test_places_beyond_32_bits():
    # a pool of more than 2^32 bytes and 2^31 values: its last pages hold what was written there
    rt = rt_module()
    n_pages = (1 << 31) // (16 * 2 * 64) + 40
    pool = lambda: torch.empty((n_pages, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    table = torch.arange(n_pages - 1, n_pages - 31, -1, dtype=torch.int32, device="cuda").view(2, 15)
    c = rt.PagedCache(pool(), pool(), table)
    seq = torch.arange(2, device="cuda").int().repeat_interleave(240)
    pos = torch.arange(240, device="cuda").int().repeat(2)
    k, v = (torch.randn((480, 2, 64), generator=gen(s), device="cuda").bfloat16() for s in (1, 2))
    c.write(k, v, seq, pos)
    kr, vr = c.read(seq, pos)
    assert torch.equal(k, kr) and torch.equal(v, vr)
    lens = [240, 227]
    q = torch.randn((2, 4, 64), generator=gen(3), device="cuda").bfloat16()
    out = c.attend(q, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    cut = lambda x: [x[:240].double(), x[240:467].double()]
    check(out, None, reference(q, cut(k), cut(v), lens), "bf16")


@pytest.mark.parametrize("slack", [1, 4000])
def test_attention_is_the_same_on_every_run_stream_and_replay(slack):
    lens, H = [3000, 1, 0, 517, 64, 2048], 4
    c, ks, vs = make_cache(lens, 2, 64, 16, "bf16", seed=8, slack=slack)
    q = torch.randn((6, H, 64), generator=gen(4), device="cuda").bfloat16()
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    first = c.attend(q, n)
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for s in side:                                                     # calls that overlap in time
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs += [c.attend(q, n) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)
    graph, lse = torch.cuda.CUDAGraph(), torch.empty((6, H), device="cuda")
    with torch.cuda.graph(graph):
        a = c.attend(q, n, lse=lse)
        b = c.attend(q, n)
    for new in (lens, [5, 700, 1, 0, 2000, 33]):                       # the lengths are read when the graph is replayed
        held = [min(x, y) for x, y in zip(new, lens)]
        n.copy_(torch.tensor(held, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        check(a, lse, reference(q, [x[:m] for x, m in zip(ks, held)], [x[:m] for x, m in zip(vs, held)], held), "bf16")
        assert torch.equal(a, b)


# ---------------------------------------------------------------- qkRMS and rotation

def turned(x, pos, freq, rot, pairs, norm, g, eps=1e-6):
    y = x
    if norm:
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        if g is not None:
            y = y * g.view(x.shape[1:])
    t = pos.double()[:, None, None] * freq[:rot // 2]
    cos, sin = torch.cos(t), torch.sin(t)
    h = rot // 2
    a, b = (y[..., :h], y[..., h:rot]) if pairs == "halves" else (y[..., 0:rot:2], y[..., 1:rot:2])
    p, q = a * cos - b * sin, a * sin + b * cos
    r = torch.cat((p, q), -1) if pairs == "halves" else torch.stack((p, q), -1).flatten(-2)
    return torch.cat((r, y[..., rot:]), -1)


def pair_size(y, rot, pairs):
    """|a| + |b| of each dimension's pair (its own magnitude where it is not rotated)."""
    y, h = y.abs(), rot // 2
    if pairs == "halves":
        s = y[..., :h] + y[..., h:rot]
        return torch.cat((s, s, y[..., rot:]), -1)
    s = y[..., 0:rot:2] + y[..., 1:rot:2]
    return torch.cat((s.repeat_interleave(2, -1), y[..., rot:]), -1)


ROTATIONS = [  # rows, heads, kv, hd, rot, pairs, norm, gains
    (1, 1, 1, 64, 64, "halves", True, True),
    (7, 3, 1, 64, 64, "neighbours", True, False),
    (33, 12, 12, 64, 32, "halves", True, True),
    (130, 5, 2, 128, 128, "halves", True, True),
    (64, 4, 4, 128, 48, "neighbours", True, True),
    (257, 16, 16, 64, 16, "halves", False, False),
    (40, 2, 0, 64, 64, "halves", True, True),
    (1001, 8, 1, 64, 0, "halves", True, True),
    (500, 6, 3, 64, 48, "halves", True, True),
    # more rows than the GPU holds warps, with heads that fill batches of four, three, two and one, and none
    (5000, 16, 16, 64, 64, "halves", True, True),
    (4001, 12, 4, 64, 64, "neighbours", True, True),
    (9001, 8, 8, 64, 32, "halves", True, False),
    (3700, 5, 3, 64, 64, "halves", True, True),
    (4500, 2, 6, 128, 128, "halves", True, True),
    (20000, 2, 1, 64, 64, "halves", True, True),
]


def rotation(case, dtype, seed=0):
    rt = rt_module()
    R, H, kv, hd, rot, pairs, norm, gains = case
    t, g = TYPES[dtype], gen(seed)
    op = rt.QkRotate(H, kv, dtype, head_dim=hd, rot_dim=rot, pairs=pairs, norm=norm)
    qkv = torch.randn((R, (H + 2 * kv) * hd + 8), generator=g, device="cuda") * torch.exp(2 * torch.randn((R, 1), generator=g, device="cuda"))
    qkv = qkv.to(t)
    q = qkv[:, :H * hd].view(R, H, hd)
    k = qkv[:, H * hd:(H + kv) * hd].view(R, kv, hd) if kv else None
    pos = torch.randint(0, 1 << 21, (R,), generator=g, device="cuda", dtype=torch.int32)
    pos[0] = 0
    gq = (1 + 0.3 * torch.randn(H * hd, generator=g, device="cuda")).to(t) if gains else None
    gk = (1 + 0.3 * torch.randn(kv * hd, generator=g, device="cuda")).to(t) if gains and kv else None
    freq = torch.tensor([10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device="cuda")
    return op, q, k, pos, gq, gk, freq


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", ROTATIONS)
def test_rotation_of_normed_queries_and_keys(case, dtype):
    R, H, kv, hd, rot, pairs, norm, gains = case
    op, q, k, pos, gq, gk, freq = rotation(case, dtype)
    qo, ko = op.forward(q, k, pos, gq, gk)
    for x, g, got in ((q, gq, qo), (k, gk, ko)):
        if x is None:
            continue
        g64 = None if g is None else g.double()
        ref = turned(x.double(), pos, freq, rot, pairs, norm, g64)
        y = turned(x.double(), pos, freq, 0, pairs, norm, g64)
        # the norm: hd squares and sums under a root, rsqrt and two products; the angle: 2^-24 of a half turn, sincospi 2 steps; two products and a sum
        err = pair_size(y, rot, pairs) * (hd / 2 + 24) * U
        assert ((got.double() - ref).abs() <= HALF_STEP[dtype] * (ref.abs() + err) + err).all()


def test_rotation_in_place_and_rows_not_in_use():
    for case in ((50, 4, 2, 64, 64, "halves", True, True), (6000, 16, 16, 64, 64, "neighbours", True, True), (4000, 12, 3, 64, 64, "halves", True, True)):
        for dtype in ("f32", "bf16"):
            op, q, k, pos, gq, gk, _ = rotation(case, dtype, seed=3)
            qo, ko = op.forward(q, k, pos, gq, gk)
            skip = torch.rand(case[0], generator=gen(5), device="cuda") < 0.3
            pos2 = torch.where(skip, -1, pos)
            q2, k2 = q.clone(), k.clone()
            a, b = op.forward(q2, k2, pos2, gq, gk, q_out=q2, k_out=k2)
            assert a is q2 and b is k2
            for got, ref, x in ((q2, qo, q), (k2, ko, k)):
                want = ref.clone()
                want[skip] = x[skip]
                assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", ROTATIONS)
def test_gradients_of_the_rotation(case, dtype):
    R, H, kv, hd, rot, pairs, norm, gains = case
    op, q, k, pos, gq, gk, freq = rotation(case, dtype, seed=1)
    g = gen(2)
    pos[R // 2] = -1 if R > 1 else 5
    used = pos >= 0
    dqo = torch.randn((R, H, hd), generator=g, device="cuda")
    dko = torch.randn((R, kv, hd), generator=g, device="cuda")
    dq, dk = torch.full_like(dqo, 7.0), torch.full_like(dko, 7.0)
    got = op.backward(q, k, pos, dqo, dko if kv else None, gq, gk, dq=dq, dk=dk if kv else None)
    # in place, and without the gains' gradients
    dq2, dk2 = dqo.clone(), dko.clone()
    op.backward(q, k, pos, dq2, dk2 if kv else None, gq, gk, dq=dq2, dk=dk2 if kv else None)
    assert torch.equal(dq2[used], dq[used]) and torch.equal(dk2[used], dk[used]) and torch.equal(dq2[~used], dqo[~used])
    for x, gain, d, dx, dg in ((q, gq, dqo, got[0], got[2]), (k, gk, dko, got[1], got[3])):
        if x is None:
            continue
        assert (dx[~used] == 7.0).all()
        x64 = x.double()[used].requires_grad_(True)
        g64 = None if gain is None else gain.double().requires_grad_(True)
        d64 = d.double()[used]
        out = turned(x64, pos[used], freq, rot, pairs, norm, g64)
        grads = torch.autograd.grad(out, [x64] + ([g64] if gain is not None and norm else []), d64)
        # dx = r (w - u mean(w u)), w = R^T d g: the errors of w and of the norm, and sums of hd terms
        r = 1 / torch.sqrt((x64 * x64).mean(-1, keepdim=True) + 1e-6) if norm else torch.ones_like(x64[..., :1])
        w = pair_size(d64, rot, pairs) * (1 if gain is None or not norm else g64.view(x64.shape[1:]).abs())
        u = (x64 * r).abs() if norm else torch.zeros_like(x64)
        err = r * (w + u * (w * u).mean(-1, keepdim=True)) * (2 * hd + 64) * U
        assert ((dx[used].double() - grads[0]).abs() <= err.detach()).all()
        if dg is not None:
            n = int(used.sum())
            ref = grads[1] if norm else torch.zeros_like(dg)
            err = (pair_size(d64, rot, pairs) * u).sum(0).reshape(-1) * (n + hd + 64) * U
            assert ((dg.double() - ref).abs() <= err.detach()).all()


# rows side by side in a warp (an odd number of them, no keys, both sizes of heads), queries and keys in one pass, in launches of their own, and calls of a few hundred rows
SHAPED_ROTATIONS = [
    (7001, 1, 1, 64, 64, "halves", True, True),
    (4999, 1, 0, 64, 32, "neighbours", True, True),
    (3001, 1, 1, 128, 128, "neighbours", True, False),
    (2503, 2, 0, 128, 64, "halves", False, False),
    (6005, 3, 1, 64, 64, "halves", True, True),
    (2501, 16, 4, 64, 64, "halves", True, True),
    (2501, 16, 4, 128, 128, "halves", True, True),
    (2402, 5, 2, 128, 128, "neighbours", True, True),
    (700, 16, 16, 64, 64, "halves", True, True),
    (900, 20, 20, 64, 48, "neighbours", True, True),
    (301, 7, 6, 128, 128, "halves", True, True),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", SHAPED_ROTATIONS)
def test_rotation_and_gradients_of_every_shape_of_pass(case, dtype):
    test_rotation_of_normed_queries_and_keys(case, dtype)
    test_gradients_of_the_rotation(case, dtype)
    # in place, with rows that are not in use
    op, q, k, pos, gq, gk, _ = rotation(case, dtype, seed=3)
    qo, ko = op.forward(q, k, pos, gq, gk)
    skip = torch.rand(case[0], generator=gen(5), device="cuda") < 0.3
    q2, k2 = q.clone(), None if k is None else k.clone()
    op.forward(q2, k2, torch.where(skip, -1, pos), gq, gk, q_out=q2, k_out=k2)
    for got, out, x in ((q2, qo, q), (k2, ko, k)):
        if x is not None:
            want = out.clone()
            want[skip] = x[skip]
            assert torch.equal(got, want)


def test_gains_of_queries_or_keys_alone_and_far_positions():
    for case in ((3000, 2, 2, 64, 64, "halves", True, True), (2500, 4, 4, 64, 64, "halves", True, True), (40, 4, 4, 64, 64, "neighbours", True, True)):
        op, q, k, pos, gq, gk, freq = rotation(case, "f32", seed=8)
        pos[:3] = torch.tensor([2 ** 31 - 1, 2 ** 31 - 2, 1], device="cuda", dtype=torch.int32)
        ones = torch.ones_like(gq)
        for a, b in ((gq, None), (None, gk)):
            got = op.forward(q, k, pos, a, b)
            want = op.forward(q, k, pos, ones if a is None else a, ones if b is None else b)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        y = turned(q.double(), pos, freq, 0, "halves", True, gq.double())
        ref = turned(q.double(), pos, freq, 64, case[5], True, gq.double())
        got = op.forward(q, k, pos, gq, None)[0]
        # far positions: 64-bit turns are off by 2^-53 of themselves, 2^31 of them by 2^-22 turns and less: 2^-19 of the pair's size
        err = pair_size(y, 64, case[5]) * ((64 / 2 + 24) * U + 2.0 ** -19)
        assert ((got.double() - ref).abs() <= HALF_STEP["f32"] * ref.abs() + 2 * err).all()


def test_gradients_of_the_rotation_against_differences():
    case = (3, 2, 1, 64, 32, "halves", True, True)
    op, q, k, pos, gq, gk, freq = rotation(case, "f32", seed=6)
    g = gen(3)
    dqo, dko = torch.randn((3, 2, 64), generator=g, device="cuda"), torch.randn((3, 1, 64), generator=g, device="cuda")
    dq, dk, dgq, dgk = op.backward(q, k, pos, dqo, dko, gq, gk)
    for x, gain, d, dx, dg in ((q, gq, dqo, dq, dgq), (k, gk, dko, dk, dgk)):
        x, gain, d = x.double(), gain.double(), d.double()
        loss = lambda a, b: float((turned(a, pos, freq, 32, "halves", True, b) * d).sum())
        for at, grad, f in ((x, dx, lambda z: loss(z, gain)), (gain, dg, lambda z: loss(x, z))):
            for s in range(3):
                step = torch.randn(at.shape, generator=g, device="cuda", dtype=torch.float64) * at.abs().mean()
                h = 1e-4
                # differences of fourth order: h^4 of the value's size, and the rounding of two 64-bit losses over h
                diff = (8 * (f(at + h * step) - f(at - h * step)) - (f(at + 2 * h * step) - f(at - 2 * h * step))) / (12 * h)
                want = float((grad.double() * step).sum())
                size = float((grad.double().abs() * step.abs()).sum())
                assert abs(diff - want) <= size * (256 * U + 1e-9), (diff, want)


def test_rotation_backward_is_captured_while_a_graph_of_the_same_leaves_lives():
    case = (300, 4, 2, 64, 64, "halves", True, True)
    op, q, k, pos, gq, gk, freq = rotation(case, "f32", seed=9)
    leaf = q.clone().requires_grad_(True)
    alive = (leaf * 2).sum()                                            # an eager autograd graph over the same data
    dqo, dko = torch.randn(300, 4, 64, device="cuda"), torch.randn(300, 2, 64, device="cuda")
    want = op.backward(leaf.detach(), k, pos, dqo, dko, gq, gk)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = op.backward(leaf.detach(), k, pos, dqo, dko, gq, gk)
    for _ in range(2):
        for x in got:
            x.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    alive.backward()
    assert (leaf.grad == 2).all()


def test_no_rows():
    rt = rt_module()
    c = rt.PagedCache.empty(4, 16, 2, 2, 2, dtype="e4m3")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    x = torch.empty((0, 2, 64), device="cuda")
    c.write(x, x, none, none)
    k, v = c.read(none, none, dtype="f32")
    assert k.shape == (0, 2, 64)
    op = rt.QkRotate(2, 2, "f32")
    op.forward(x, x, none)
    dq, dk, dgq, dgk = op.backward(x, x, none, x, x, torch.ones(128, device="cuda"), torch.ones(128, device="cuda"))
    assert dq.shape == (0, 2, 64) and (dgq == 0).all() and (dgk == 0).all()


def test_tensors_that_are_refused():
    rt = rt_module()
    c = rt.PagedCache.empty(4, 16, 2, 2, 2)
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    q = torch.zeros((2, 4, 64), device="cuda", dtype=torch.bfloat16)
    refused = [lambda: c.attend(q.cpu(), n), lambda: c.attend(q, n.cpu()), lambda: c.attend(q, n.long()), lambda: c.attend(q[:1], n), lambda: c.attend(q.half(), n),
               lambda: c.attend(q[:, :3], n), lambda: c.attend(q.transpose(1, 2).contiguous().transpose(1, 2), n), lambda: c.attend(q, n, k_own=q[:, :2]),
               lambda: c.attend(q, n, out=q), lambda: c.attend(q, n, out=torch.empty((2, 4, 64), device="cuda")), lambda: c.attend(q, n, lse=torch.empty((2, 4), device="cuda").double()),
               lambda: c.attend(q, n, alibi_slopes=torch.ones(3, device="cuda")), lambda: c.write(q[:, :2], q[:, :2], n, n[:1]),
               lambda: c.write(q, q, n, n), lambda: c.write(q[:, :2], q[:, :2].float(), n, n), lambda: c.read(n, n, k=torch.empty((2, 2, 64), device="cuda")),
               lambda: rt.PagedCache(c.k, c.v.transpose(2, 3), c.page_table), lambda: rt.PagedCache(c.k, c.v, c.page_table.long()),
               lambda: rt.PagedCache(c.k, c.v, c.page_table, c.k.view(torch.uint8)), lambda: rt.PagedCache(c.k.cpu(), c.v.cpu(), c.page_table.cpu()),
               lambda: rt.QkRotate(4, 2).forward(q, q[:, :2], n.long()), lambda: rt.QkRotate(4, 2).forward(q.float(), q[:, :2].float(), n),
               lambda: rt.QkRotate(4, 2, rot_dim=40), lambda: rt.QkRotate(4, 2).backward(q, q[:, :2], n, q, q[:, :2].float())]
    for f in refused:
        with pytest.raises(rt.RtError):
            f()


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("cache", ["f32", "e4m3"])
def test_a_recurrent_layer_goes_on_from_pages_of_ragged_length(cache):
    """A batch that one layer has prefilled together goes on from different lengths: its pairs move into pages, and each step norms (no rotation: rot_dim 0)
    queries and keys, attends over the pages and the temporary pair, and writes the persistent pair of the layer's output."""
    from oracle import RTConfig, RTWeights, layer_seq
    from paper_2604_21215_b200 import inputs
    rt = rt_module()
    d, H, dff, B, N = 128, 2, 512, 4, 60
    slopes = [0.25, 0.0625]
    data = inputs.make_inputs(inputs.Workload("pages", 1, B, N, d, H, dff, "f32"), seed=5)
    lw = dict(data["layers"][0], alibi_slopes=slopes)
    rng = np.random.default_rng(6)
    for n in ("g_attn", "g_mlp", "g_kv", "g_q", "g_k"):
        lw[n] = (1 + 0.2 * rng.standard_normal(d)).astype(np.float32).astype(np.float64)
    x = data["x"]
    ocfg = RTConfig(d, H, 64, dff, alibi_slopes=slopes)
    z_ref, _, _ = layer_seq(ocfg, RTWeights(**{n: v for n, v in lw.items() if n != "alibi_slopes"}), x)
    layer = rt.Layer(d, H, dff, dtype="f32", leaf=16)
    layer.set_weights(lw)
    lens, steps = [0, 1, 37, 56], 4                                     # what each sequence keeps of the prefill, and how far it goes on
    layer.prefill(x[:, :56], N_max=56)
    c = rt.PagedCache.empty(24, 16, H, B, 5, dtype=cache)
    c.page_table.copy_(torch.randperm(24, generator=torch.Generator().manual_seed(3))[:20].view(B, 5).int())
    seq = torch.arange(B, device="cuda").int().repeat(56)               # rows of the layer's cache: position-major
    pos = torch.arange(56, device="cuda").int().repeat_interleave(B)
    keep = torch.where(pos < torch.tensor(lens, device="cuda").int()[seq.long()], pos, -1)
    c.write(layer.k_cache.view(56 * B, d), layer.v_cache.view(56 * B, d), seq, keep)

    w = {n: torch.tensor(lw[n], device="cuda") for n in lw}
    g32 = {n: w[n].float() for n in ("g_q", "g_k")}
    rot = rt.QkRotate(H, H, "f32", rot_dim=0)
    rms = lambda u, g: u / torch.sqrt((u * u).mean(-1, keepdim=True) + 1e-6) * g
    slope_t = torch.tensor(slopes, device="cuda")
    batch = torch.arange(B, device="cuda").int()
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    worst = 0.0
    for s in range(steps):
        xi = torch.tensor(np.stack([x[b, lens[b] + s] for b in range(B)]), device="cuda")
        u = rms(xi, w["g_attn"])
        q, kt, vt = ((u @ w[m].T).float() for m in ("w_q", "w_k", "w_v"))
        q, kt = rot.forward(q, kt, n, g32["g_q"], g32["g_k"])
        a = c.attend(q.view(B, H, 64), n, k_own=kt.view(B, H, 64), v_own=vt.view(B, H, 64), alibi_slopes=slope_t)
        h = xi + a.double().view(B, d) @ w["w_o"].T
        z = h + torch.nn.functional.gelu(rms(h, w["g_mlp"]) @ w["w_up"].T) @ w["w_down"].T
        uz = rms(z, w["g_kv"])
        kp, vp = ((uz @ w[m].T).float() for m in ("w_k", "w_v"))
        _, kp = rot.forward(kp, kp, n, g32["g_q"], g32["g_k"])
        c.write(kp.view(B, H, 64), vp.view(B, H, 64), batch, n)
        ref = np.stack([z_ref[b, lens[b] + s] for b in range(B)])
        worst = max(worst, float((z.cpu().numpy() - ref).__abs__().max() / np.abs(ref).max()))
        n += 1
    torch.cuda.synchronize()
    assert c.status() == rt.RT_OK
    # fp32: the library's own tolerance for a layer.  e4m3: keys and values off by up to 2^-4 each; the attention averages, the layer adds it to x: the
    # difference stays below the rounding of a single pair
    assert worst <= (1e-4 if cache == "f32" else 2.0 ** -4), worst


def test_first_calls_may_be_captured():
    # in a process of its own, where no kernel has run before
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2604_21215_b200 import rt
c = rt.PagedCache.empty(64, 16, 2, 2, 32, head_dim=128, dtype="e4m3")
c.page_table.copy_(torch.arange(64).view(2, 32).int())
n = torch.tensor([300, 17], dtype=torch.int32, device="cuda")
q, kv = torch.randn(2, 6, 128, device="cuda"), torch.randn(2, 2, 128, device="cuda")
g, seq = torch.ones(6 * 128, device="cuda"), torch.arange(2, device="cuda").int()
op = rt.QkRotate(6, 2, "f32", head_dim=128)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
def step():
    qr, kr = op.forward(q, kv, n, g, g[:256])
    c.write(kr, kv, seq, n)
    out = c.attend(qr, n, k_own=kr, v_own=kv)
    k, v = c.read(seq, n, dtype="f32")
    return (out, k, v) + op.backward(q, kv, n, qr, kr, g, g[:256])
with torch.cuda.graph(graph):
    got = step()
graph.replay()
torch.cuda.synchronize()
want = step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, want)) and c.status() == 0
print("captured")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("cache,n", [("e4m3", 90000), ("bf16", 40000)])
def test_sums_of_long_sequences_are_added_in_fp32(cache, n):
    """Queries of zeros weigh all pairs alike and values are positive, so an output is the mean of its values, and its error in fp32 that of the sums: half a step for each
    unit that a warp adds up, a few steps inside a unit, the joined parts.  (A tensor core that accumulated a whole piece would lose up to a step with every product.)
    The bf16 output then lies between the roundings of the two ends."""
    rt = rt_module()
    B, H, hd, page = 8, 16, 64, 64
    m = -(-n // page)
    c = rt.PagedCache.empty(B * m, page, H, B, m, head_dim=hd, dtype=cache)
    c.page_table.copy_(torch.arange(B * m).flip(0).view(B, m).int())
    g = gen(12)
    part = torch.rand((1, H, 1, hd), generator=g, device="cuda")        # how often a dimension is large: the means cover the steps of bf16
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    want = []
    for b in range(B):
        pages = slice((B - 1 - b) * m, (B - b) * m)                     # (flipped: the sequence's pages from the last to the first)
        large = torch.rand((m, H, page, hd), generator=g, device="cuda") < part
        e = torch.randint(-20, 1, (m, H, page), generator=g, device="cuda")
        if cache == "e4m3":
            c.v.view(torch.uint8)[pages] = torch.where(large, 0x3f, 0x38).to(torch.uint8)       # 1.875, 1
            c.v_exp[pages] = (127 + e).to(torch.uint8)
            v = torch.where(large, 1.875, 1.0).double() * (2.0 ** e.double())[..., None]
        else:
            v = torch.where(large, 1.9921875, 1.0) * (2.0 ** e.float())[..., None]
            c.v[pages] = v.bfloat16()
            v = v.double()
        v = v.flip(0).transpose(0, 1).reshape(H, m * page, hd)[:, :n]
        want.append(v.mean(1))
    out = c.attend(torch.zeros((B, H, hd), dtype=torch.bfloat16, device="cuda"), lens).double()
    o = torch.stack(want)
    unit, warps = 64 if cache == "e4m3" else 32, 148 * 12
    per_warp, parts = B * H * -(-n // unit) / warps, warps / (B * H) + 2
    err = (per_warp + parts + 16 + 24) * U                              # 16: four products of a unit, four half steps each; 24: the division and the like
    low, high = (x.float().bfloat16().double() for x in (o * (1 - err), o * (1 + err)))
    assert ((out >= low) & (out <= high)).all(), int(((out < low) | (out > high)).sum())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
def test_values_keep_their_scale_beside_scores_of_any_size(cache, hd, dtype):
    """Scores that are whole powers of two: one pair gives its value, two pairs of one key the mean of their values however large the score and however small the values;
    a third pair, far below, has no weight.  Weights are good to 2^-20, and the values are exact in both types of pages."""
    rt = rt_module()
    c = rt.PagedCache.empty(3, 16, 1, 3, 1, head_dim=hd, dtype=cache)
    c.page_table.copy_(torch.arange(3).view(3, 1).int())
    at = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    seq, pos = at(0, 1, 1, 2, 2, 2), at(0, 0, 1, 0, 1, 2)
    for score in (1.0, 2.0 ** 10, 2.0 ** 17, 2.0 ** 23, -2.0 ** 24, 2.0 ** 28, -2.0 ** 28, 2.0 ** 40):
        for e in (-120, -100, -30, -8, -3, 0, 20, 60, 110):
            k = torch.zeros((6, 1, hd), device="cuda")
            k[:, 0, 0] = 1.0
            k[5, 0, 0] = -1.0 if score > 0 else 2.0                     # 2 |score| or |score| below the others
            far = abs(score) > 200
            v = (1.0 + torch.arange(6 * hd, device="cuda").remainder(7).float()).view(6, 1, hd) * 2.0 ** e
            v[[2, 4]] *= 0.125                                          # (another scale)
            v[5] *= 2.0 ** 10
            c.write(k, v, seq, pos)
            kr, vr = c.read(seq, pos, dtype="f32")
            assert torch.equal(kr, k) and torch.equal(vr, v)
            q = torch.zeros((3, 1, hd), device="cuda", dtype=TYPES[dtype])
            q[:, 0, 0] = score
            lse = torch.empty((3, 1), device="cuda")
            out = c.attend(q, at(1, 2, 3 if far else 2), scale=1.0, lse=lse).double()[:, 0]
            v = v.double()[:, 0]
            want = torch.stack((v[0], (v[1] + v[2]) / 2, (v[3] + v[4]) / 2))
            assert ((out - want).abs() <= (2.0 ** -20 + HALF_STEP[dtype]) * want).all(), (score, e)
            assert ((lse.double()[:, 0] - score - torch.tensor([0.0, math.log(2.0), math.log(2.0)], device="cuda")).abs() <= 4 * U * abs(score) + 2.0 ** -20).all()


def same_numbers(got, want, err):
    """NaN and infinities where they belong, all else within err (of the finite ones)."""
    got, fine = got.double(), torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    odd = ~fine & ~torch.isnan(want)
    assert torch.equal(got[odd], want[odd])
    assert ((got - want).abs() <= err)[fine].all()


# rows side by side, queries and keys in passes of their own and mixed, small calls; nothing rotated, and parts of a head
PARTLY_ROTATED = [(3, 1, 1, 64, 0), (40, 2, 1, 64, 32), (7001, 1, 1, 64, 16), (5000, 16, 16, 64, 32), (3700, 5, 3, 64, 48), (2402, 5, 2, 128, 64), (300, 4, 4, 128, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("shape", PARTLY_ROTATED)
def test_infinities_and_nan_stay_in_their_pair(shape, pairs, norm, dtype):
    # dimensions that are not rotated have no partner; a rotated one has its own
    R, H, kv, hd, rot = shape
    op, q, k, pos, gq, gk, freq = rotation((R, H, kv, hd, rot, pairs, norm, norm), dtype, seed=4)
    g = gen(6)
    bad = torch.tensor([math.inf, -math.inf, math.nan], device="cuda")
    for x in (q, k):
        n = max(1, R // 50)
        x[torch.randint(0, R, (n,), generator=g, device="cuda"), torch.randint(0, x.shape[1], (n,), generator=g, device="cuda"),
          torch.randint(0, hd, (n,), generator=g, device="cuda")] = bad[torch.randint(0, 3, (n,), generator=g, device="cuda")].to(x.dtype)
        x[0, 0, hd - 1] = math.inf                                      # (the last dimension, next to one that is not rotated either)
    got = op.forward(q, k, pos, gq, gk)
    for x, gain, y in zip((q, k), (gq, gk), got):
        g64 = None if gain is None else gain.double()
        want = turned(x.double(), pos, freq, rot, pairs, norm, g64)
        err = pair_size(turned(x.double(), pos, freq, 0, pairs, norm, g64), rot, pairs) * (hd / 2 + 24) * U
        same_numbers(y, want.to(y.dtype).double(), HALF_STEP[dtype] * 2 * (want.abs() + err) + err)
        if not norm:
            assert torch.equal(torch.nan_to_num(y[..., rot:]), torch.nan_to_num(x[..., rot:]))       # what is not rotated is copied

    # the gradients: one infinity in some heads
    q, k = rotation((R, H, kv, hd, rot, pairs, norm, norm), dtype, seed=4)[1:3]
    d = [torch.randn((R, h, hd), generator=g, device="cuda") for h in (H, kv)]
    for x in d:
        x[0, 0, hd - 1] = math.inf
        x[R // 2, x.shape[1] - 1, hd // 2 if rot <= hd // 2 else hd - 2] = -math.inf
    got = op.backward(q, k, pos, d[0], d[1], gq, gk)
    for x, gain, dy, dx, dg in zip((q, k), (gq, gk), d, got[:2], got[2:]):
        x, w = x.double(), turned(dy.double(), -pos, freq, rot, pairs, False, None)
        size = pair_size(torch.where(torch.isfinite(dy), dy.double(), 0.0), rot, pairs)
        if not norm:
            same_numbers(dx, w, size * 64 * U)
            continue
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        u, wg = x * r, w * gain.double().view(x.shape[1:])
        want = r * (wg - u * (wg * u).mean(-1, keepdim=True))
        s = size * gain.double().abs().view(x.shape[1:])
        same_numbers(dx, want, r * (s + u.abs() * (s * u.abs()).mean(-1, keepdim=True)) * (2 * hd + 64) * U)
        same_numbers(dg, (w * u).sum(0).reshape(-1), (size * u.abs()).sum(0).reshape(-1) * (R + hd + 64) * U)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("slack", [0, 40])
def test_8_bit_pages_that_do_not_exist_and_lengths_that_are_cut(slack, hd, dtype):
    # a unit of 64 positions has four pages of 16: any of them may be missing, in the middle and at the ragged end
    rt = rt_module()
    lens, H, kv = [70, 330, 64], 4, 2
    c, ks, vs = make_cache(lens, kv, hd, 16, "e4m3", seed=16, slack=slack)
    q = torch.randn((3, H, hd), generator=gen(4), device="cuda").to(TYPES[dtype])
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    lse = torch.empty((3, H), device="cuda")
    check(c.attend(q, n, lse=lse), lse, reference(q, ks, vs, lens), dtype)
    torch.cuda.synchronize()
    assert c.status() == rt.RT_OK
    for missing, bad in (([4], -1), ([5], c.k.shape[0]), ([6], 2 ** 31 - 1), ([7], -2 ** 31), ([8, 9, 10, 11], -1), ([20], -7), ([0, 3, 13], 1 << 30), (list(range(21)), -1)):
        old = c.page_table[1].clone()
        c.page_table[1, missing] = bad
        out = c.attend(q, n, lse=lse)
        torch.cuda.synchronize()
        assert c.status() == rt.RT_ERR_INVALID_ARG
        c.page_table[1] = old
        c.clear_status()
        keep = torch.tensor([j for j in range(330) if j // 16 not in missing], dtype=torch.long, device="cuda")
        cut = lambda x: [x[0], x[1][keep], x[2]]                            # the pairs of those pages have no weight
        check(out, lse, reference(q, cut(ks), cut(vs), lens), dtype)
    if slack == 0:                                                        # a length beyond the table is cut to it: 336 positions, the last six written here
        pos = torch.arange(330, 336, dtype=torch.int32, device="cuda")
        x = torch.randn((6, kv, hd), generator=gen(8), device="cuda")
        c.write(x, x, torch.ones_like(pos), pos)
        x = c.read(torch.ones_like(pos), pos, dtype="f32")[0].double()
        out = c.attend(q, torch.tensor([70, 2 ** 31 - 1, 64], dtype=torch.int32, device="cuda"), lse=lse)
        torch.cuda.synchronize()
        assert c.status() == rt.RT_ERR_INVALID_ARG
        check(out, lse, reference(q, [ks[0], torch.cat((ks[1], x)), ks[2]], [vs[0], torch.cat((vs[1], x)), vs[2]], lens), dtype)


@pytest.mark.parametrize("cache,dtype", [("e4m3", "bf16"), ("e4m3", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("hd,slack", [(64, 0), (64, 4000), (128, 0), (128, 4000)])
def test_a_nan_that_is_attended_to_stays_in_its_head(hd, slack, cache, dtype):
    # such heads are evaluated position by position: their other dimensions, and all other heads, are as good as ever
    lens, H, kv = [300, 41, 700, 90], 6, 3
    c, ks, vs = make_cache(lens, kv, hd, 16, cache, seed=18, slack=slack)
    raw = lambda pool: pool.view(torch.uint8) if cache == "e4m3" else pool
    nan = 0x7f if cache == "e4m3" else math.nan
    place = lambda b, j: (int(c.page_table[b, j // 16]), j % 16)
    marks = [(0, 1, 130, 5, "k"), (1, 0, 40, 9, "v"), (2, 2, 699, hd - 1, "v"), (2, 0, 3, 0, "v"), (3, 1, 0, 1, "k")]
    for b, h, j, d, which in marks:
        p, o = place(b, j)
        raw(c.k if which == "k" else c.v)[p, h, o, d] = nan
        (ks if which == "k" else vs)[b][j, h, d] = math.nan
    q = torch.randn((4, H, hd), generator=gen(4), device="cuda").to(TYPES[dtype])
    lse = torch.empty((4, H), device="cuda")
    out = c.attend(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), lse=lse)
    o, l, eo, el = reference(q, ks, vs, lens)
    assert torch.equal(torch.isnan(out.float()), torch.isnan(o)) and torch.equal(torch.isnan(lse), torch.isnan(l))
    assert int(torch.isnan(o).all(-1).sum()) == 4 and int(torch.isnan(o).sum()) == 4 * hd + 6        # two query heads on each head of the cache
    # (the bound of a NaN dimension is NaN: nothing to compare there; the bounds of finite ones come from finite values)
    fine = ~torch.isnan(o)
    bound = HALF_STEP[dtype] * (o.abs() + eo) + eo + 1e-30
    assert ((out.double() - o).abs() <= bound)[fine].all()
    assert ((lse.double() - l).abs() <= el)[~torch.isnan(l)].all()
