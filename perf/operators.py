"""Caches in pages and what belongs to them, as cases that can be timed and whose outputs can be compared.

A server that decodes ragged batches keeps the pairs of its sequences in pages of a pool, in the storage type or in 8
bits; a case is one call of one of the operators around such a cache:

    attend     attention of one new token of every sequence over its cached pairs (and, for a Recurrent Transformer
               layer, over the token's own temporary pair)
    write      rows of keys and values into their places in the pages, quantised there for an 8-bit cache
    read       rows of keys and values out of the pages, as the values they stand for
    rotate     qkRMS of queries and keys for each head, and the rotation by the position, in one pass
    rotgrad    its gradients: of queries, keys and gains

`own` false: the plain forms in elementary torch operations.  `own` true: the package's operators.
Pools are [pages, kv_heads, page, head_dim]; an e4m3 pool has an 8-bit exponent (bias 127) for each row of a head.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
_SIZE = {"f32": 4, "bf16": 2, "e4m3": 1}


def _case(op, dtype, cache, B, lo, hi, heads, kv=None, hd=64, page=16, alibi=False, pair=False, gains=True, rot=None, pairs="halves",
          name=None):
    """B sequences with lo to hi positions each.  cache: type of the pages.  pair: with the token's own temporary pair."""
    c = {"op": op, "dtype": dtype, "cache": cache, "B": B, "lo": lo, "hi": hi, "heads": heads, "kv": heads if kv is None else kv,
         "hd": hd, "page": page, "alibi": alibi, "pair": pair, "gains": gains, "rot": hd if rot is None else rot, "pairs": pairs}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user in the middle of an answer: a call for each layer and token, where latency counts
        _case("attend", "bf16", "bf16", 1, 1024, 1024, 16, alibi=True, pair=True, name="attend_one_user"),
        # a batch of requests of all ages at the width of the 150M models, one of them empty so far
        _case("attend", "bf16", "bf16", 24, 0, 4096, 12, pair=True, name="attend_ragged_batch"),
        # long documents in an 8-bit cache, the largest case
        _case("attend", "bf16", "e4m3", 16, 12001, 32768, 16, page=64, name="attend_long_e4m3"),
        # four query heads on each head of the cache, wide heads
        _case("attend", "bf16", "bf16", 40, 517, 8192, 16, kv=4, hd=128, page=32, name="attend_shared_heads"),
        # one step of a full batch into an 8-bit cache
        _case("write", "bf16", "e4m3", 16, 300, 1024, 16, name="write_step_e4m3"),
        # the prompts of a full batch into an 8-bit cache
        _case("write", "bf16", "e4m3", 16, 1999, 2048, 16, page=64, name="write_prompt_e4m3"),
        # a short prefix out of the cache, for a second request that begins with it
        _case("read", "bf16", "bf16", 1, 257, 257, 12, name="read_prefix"),
        # the whole cache of a batch as bf16 rows, for a parallel sweep over them
        _case("read", "bf16", "e4m3", 8, 3001, 4096, 16, page=64, name="read_batch_e4m3"),
        # queries and keys of one step of a full batch
        _case("rotate", "bf16", "bf16", 16, 1, 1, 16, name="rotate_step"),
        # queries and keys of the prompts of a batch
        _case("rotate", "bf16", "bf16", 8, 4001, 4096, 16, name="rotate_prompt"),
        # a training step of a small model in fp32, a part of each head rotated, neighbours paired
        _case("rotgrad", "f32", "f32", 4, 256, 256, 2, rot=32, pairs="neighbours", name="rotgrad_small_f32"),
        # a training batch at the width of the 300M models
        _case("rotgrad", "bf16", "bf16", 8, 4001, 4096, 16, name="rotgrad_batch"),
    ]


def _spread(rng, lo, hi):
    """A whole number from [lo, hi], evenly spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attend", "attend", "attend", "write", "read", "rotate", "rotgrad"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    hd = rng.choice((64, 64, 64, 128))
    kv = rng.choice((1, 2, 3, 4, 6, 8, 12, 16)) if hd == 64 else rng.choice((1, 2, 4, 8))
    page = rng.choice((16, 32, 64, 128, 256))
    if op in ("rotate", "rotgrad"):
        hi = _spread(rng, 1, 4096)
        B = _spread(rng, 1, max(1, 30000 // hi))
        return _case(op, dtype, dtype, B, max(1, hi // 2), hi, kv * rng.choice((1, 1, 2, 4)) if kv <= 4 else kv, kv=kv, hd=hd,
                     gains=rng.random() < 0.6, rot=rng.choice((hd, hd, hd // 2, 16)), pairs=rng.choice(("halves", "neighbours")))
    cache = rng.choice((dtype, "e4m3", "e4m3"))
    hi = _spread(rng, 1, 32768)
    most = 16 * 20000 * 1024 // (hi * kv * hd * (1 if cache == "e4m3" else 2 if cache == "bf16" else 4))
    if op != "attend":
        most = min(most, 30000 * 1024 // (hi * kv * hd))
    B = _spread(rng, 1, max(1, min(200, most)))
    lo = rng.choice((0, 1, hi // 2, hi)) if op == "attend" else max(1, rng.choice((1, hi // 2, hi)))
    return _case(op, dtype, cache, B, min(lo, hi), hi, kv * rng.choice((1, 1, 2, 3, 4, 8)), kv=kv, hd=hd, page=page,
                 alibi=rng.random() < 0.4, pair=rng.random() < 0.5)


def _lengths(c):
    """The sequences' lengths, spread over [lo, hi], the first one hi."""
    return [c["hi"] - (b * 2654435769 % 2 ** 32) * (c["hi"] - c["lo"] + 1) // 2 ** 32 for b in range(c["B"])]


def _rows(c):
    """(sequence, position) of the rows of a call that is not `attend`: a whole prompt each, or one step."""
    n = _lengths(c)
    if c["op"] == "write" and c["hi"] < 1500 and c["B"] > 1:                # one new token behind what each sequence has
        return list(range(c["B"])), [x - 1 for x in n]
    return [b for b, x in enumerate(n) for _ in range(x)], [i for x in n for i in range(x)]


def _pool(c, gen, dev, n_pages):
    shape = (n_pages, c["kv"], c["page"], c["hd"])
    if c["cache"] != "e4m3":
        return torch.randn(shape, generator=gen, device=dev).to(_TYPES[c["cache"]]), None
    code = (100.0 * torch.randn(shape, generator=gen, device=dev)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return code, torch.randint(119, 122, shape[:3], generator=gen, device=dev, dtype=torch.uint8)


def prepare(case, seed):
    c = case
    dev = torch.device("cuda", 0) if torch.cuda.is_available() else torch.device("cpu")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    tdt, H, kv, hd = _TYPES[c["dtype"]], c["heads"], c["kv"], c["hd"]
    st = {"case": c}
    if c["op"] in ("rotate", "rotgrad"):
        pos = _rows(c)[1] if c["hi"] > 1 else [(1009 * b) % 4096 for b in range(c["B"])]
        R, h = len(pos), c["rot"] // 2
        # what the three projections of a layer leave in one array: queries and keys are views of its rows
        qkv = rand(R, (H + 2 * kv) * hd).to(tdt)
        st["q"], st["k"] = qkv[:, :H * hd].view(R, H, hd), qkv[:, H * hd:(H + kv) * hd].view(R, kv, hd)
        st["pos"] = torch.tensor(pos, dtype=torch.int32, device=dev)
        st["freq"] = torch.tensor([10000.0 ** (-i / h) for i in range(h)], dtype=torch.float64, device=dev)
        for n, heads in (("g_q", H), ("g_k", kv)):
            st[n] = (1.0 + 0.1 * rand(heads * hd)).to(tdt) if c["gains"] else None
        if c["op"] == "rotgrad":
            st["dq_out"], st["dk_out"] = rand(R, H, hd), rand(R, kv, hd)
        if own:
            from paper_2604_21215_b200 import rt
            st["rot"] = rt.QkRotate(H, kv, c["dtype"], head_dim=hd, rot_dim=c["rot"], base=10000.0, pairs=c["pairs"], rms_eps=1e-6)
        return st
    n, P = _lengths(c), c["page"]
    room = 1 if c["op"] == "attend" else 0                                   # an attended cache has room for the new token
    need = [-(-(x + room) // P) for x in n]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
    table = torch.full((c["B"], max(max(need), 1)), -1, dtype=torch.int32)   # (entries behind a sequence's pages name no page)
    table, at, order = table.numpy(), 0, order.cpu().numpy()
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    st["table"] = torch.from_numpy(table).to(dev)
    st["k"], st["ke"] = _pool(c, gen, dev, n_pages)
    st["v"], st["ve"] = _pool(c, gen, dev, n_pages)
    if c["op"] == "attend":
        st["q"] = rand(c["B"], H, hd).to(tdt)
        st["lens"] = torch.tensor(n, dtype=torch.int32, device=dev)
        st["k_own"], st["v_own"] = (rand(c["B"], kv, hd).to(tdt), rand(c["B"], kv, hd).to(tdt)) if c["pair"] else (None, None)
        st["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device=dev) if c["alibi"] else None
        st["lse"] = torch.empty((c["B"], H), dtype=torch.float32, device=dev)
    else:
        seq, pos = _rows(c)
        st["seq"] = torch.tensor(seq, dtype=torch.int32, device=dev)
        st["pos"] = torch.tensor(pos, dtype=torch.int32, device=dev)
        if c["op"] == "write":
            st["k_rows"], st["v_rows"] = rand(len(seq), kv, hd).to(tdt), (0.5 * rand(len(seq), kv, hd)).to(tdt)
    if own:
        from paper_2604_21215_b200 import rt
        st["cache"] = rt.PagedCache(st["k"], st["v"], st["table"], st["ke"], st["ve"])
    return st


# ---------------------------------------------------------------- the plain forms

def _scale_of(e):
    return (e.to(torch.int32) << 23).view(torch.float32)                      # (the exponents are at least 1)


def _gathered(pool, e, table):
    """The pages of every sequence in fp32: [B, kv, positions, head_dim]."""
    at = table.clamp(min=0).long()
    x = (pool.view(torch.uint8)[at].view(pool.dtype) if e is not None else pool[at]).float()
    if e is not None:
        x = x * _scale_of(e[at])[..., None]
    B, m, kv, P, hd = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(B, kv, m * P, hd)


def _plain_attend(st):
    c = st["case"]
    B, H, kv, hd = c["B"], c["heads"], c["kv"], c["hd"]
    k, v = _gathered(st["k"], st["ke"], st["table"]), _gathered(st["v"], st["ve"], st["table"])
    j = torch.arange(k.shape[2], device=k.device)
    live = j[None, :] < st["lens"][:, None]                                   # [B, positions]
    v = torch.where(live[:, None, :, None], v, 0.0)
    q = st["q"].float().view(B, kv, H // kv, hd)
    a = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(hd)                    # [B, kv, group, positions]
    at = st["lens"] if c["pair"] else st["lens"] - 1                          # the query's position
    if st["slopes"] is not None:
        a = a - st["slopes"].view(1, kv, H // kv, 1) * (at[:, None] - j[None, :]).float()[:, None, None, :]
    a = torch.where(live[:, None, None, :], a, -math.inf)
    if c["pair"]:
        own_a = (q * st["k_own"].float()[:, :, None, :]).sum(-1, keepdim=True) / math.sqrt(hd)
        a = torch.cat((a, own_a), -1)
        v = torch.cat((v, st["v_own"].float()[:, :, None, :]), 2)
    m = a.amax(-1, keepdim=True)
    p = torch.exp(a - torch.where(m == -math.inf, 0.0, m))
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(l == 0.0, 1.0, l)                    # a sequence without any pair gets zeros
    return o.reshape(B, H, hd).to(_TYPES[c["dtype"]]), (m + torch.log(l)).reshape(B, H)


def _quantised(x):
    """e4m3 codes of rows in fp32, and the exponents of their scales: the smallest power of two that brings the row within 448."""
    fine = torch.isfinite(x)
    most = torch.where(fine, x.abs(), 0.0).amax(-1)
    f, e = torch.frexp(most)                                                  # most = f 2^e, 1/2 <= f < 1; 448 = 0.875 2^9
    e = torch.where(most > 0.0, e - 9 + (f > 0.875), -126).clamp(min=-126)
    code = torch.where(fine, torch.ldexp(x, -e[..., None]), math.nan).to(torch.float8_e4m3fn)
    return code, (e + 127).to(torch.uint8)


def _plain_write(st):
    P = st["case"]["page"]
    keep = st["pos"] >= 0
    seq, pos = st["seq"][keep].long(), st["pos"][keep].long()
    page, off = st["table"][seq, pos // P].long(), pos % P
    for rows, pool, e in ((st["k_rows"], st["k"], st["ke"]), (st["v_rows"], st["v"], st["ve"])):
        if e is None:
            pool[page, :, off] = rows[keep].to(pool.dtype)
        else:
            code, ex = _quantised(rows[keep].float())
            pool.view(torch.uint8)[page, :, off] = code.view(torch.uint8)
            e[page, :, off] = ex
    return _pools(st)


def _pools(st):
    if st["ke"] is None:
        return st["k"], st["v"]
    return st["k"], st["v"], st["ke"].view(torch.float8_e8m0fnu), st["ve"].view(torch.float8_e8m0fnu)


def _plain_read(st):
    c = st["case"]
    seq, pos = st["seq"].long(), st["pos"].long()
    page, off = st["table"][seq, pos // c["page"]].long(), pos % c["page"]
    if st["ke"] is None:
        return tuple(p[page, :, off].float().to(_TYPES[c["dtype"]]) for p in (st["k"], st["v"]))
    return tuple((p.view(torch.uint8)[page, :, off].view(p.dtype).float() * _scale_of(e[page, :, off])[..., None]).to(_TYPES[c["dtype"]])
                 for p, e in ((st["k"], st["ke"]), (st["v"], st["ve"])))


def _angles(st):
    t = st["pos"].double()[:, None] * st["freq"]                              # (far positions need the 64 bits)
    return torch.cos(t).float()[:, None, :], torch.sin(t).float()[:, None, :]


def _turned(y, cos, sin, c):
    """The rotated part's pairs turned by the angles, the rest of each head as it is."""
    r, h = c["rot"], c["rot"] // 2
    a, b = (y[..., :h], y[..., h:r]) if c["pairs"] == "halves" else (y[..., 0:r:2], y[..., 1:r:2])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat((a, b), -1) if c["pairs"] == "halves" else torch.stack((a, b), -1).flatten(-2)
    return torch.cat((turned, y[..., r:]), -1)


def _plain_rotate(st):
    c = st["case"]
    cos, sin = _angles(st)
    out = []
    for n, g in (("q", "g_q"), ("k", "g_k")):
        x = st[n].float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        if st[g] is not None:
            y = y * st[g].float().view(x.shape[1:])
        out.append(_turned(y, cos, sin, c).to(_TYPES[c["dtype"]]))
    return tuple(out)


def _plain_rotgrad(st):
    c = st["case"]
    cos, sin = _angles(st)
    grads, gains = [], []
    for n, g, d in (("q", "g_q", "dq_out"), ("k", "g_k", "dk_out")):
        x = st[n].float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        u = x * r
        dy = _turned(st[d], cos, -sin, c)                                     # the rotation backwards
        if st[g] is not None:
            gains.append((dy * u).sum(0).reshape(-1))
            dy = dy * st[g].float().view(x.shape[1:])
        grads.append(r * (dy - u * (dy * u).mean(-1, keepdim=True)))
    return tuple(grads + gains)


def run(state):
    c = state["case"]
    if not own:
        return {"attend": _plain_attend, "write": _plain_write, "read": _plain_read, "rotate": _plain_rotate, "rotgrad": _plain_rotgrad}[c["op"]](state)
    if c["op"] == "attend":
        out = state["cache"].attend(state["q"], state["lens"], k_own=state["k_own"], v_own=state["v_own"], alibi_slopes=state["slopes"],
                                    lse=state["lse"])
        return out, state["lse"]
    if c["op"] == "write":
        state["cache"].write(state["k_rows"], state["v_rows"], state["seq"], state["pos"])
        return _pools(state)
    if c["op"] == "read":
        return state["cache"].read(state["seq"], state["pos"], dtype=c["dtype"])
    if c["op"] == "rotate":
        return state["rot"].forward(state["q"], state["k"], state["pos"], state["g_q"], state["g_k"])
    dq, dk, dg_q, dg_k = state["rot"].backward(state["q"], state["k"], state["pos"], state["dq_out"], state["dk_out"], state["g_q"], state["g_k"])
    return (dq, dk, dg_q, dg_k) if c["gains"] else (dq, dk)


def work(case):
    c = case
    H, kv, hd, e, s = c["heads"], c["kv"], c["hd"], _SIZE[c["dtype"]], _SIZE[c["cache"]]
    row = kv * (hd * s + (1 if c["cache"] == "e4m3" else 0))                  # a position's keys, or values, in the cache
    if c["op"] == "attend":
        pairs = sum(_lengths(c)) + (c["B"] if c["pair"] else 0)
        nbytes = 2 * sum(_lengths(c)) * row + c["B"] * (H * (2 * hd * e + 4) + (2 * kv * hd * e if c["pair"] else 0))
        return {"bytes": nbytes, "flops": 4 * pairs * H * hd}
    if c["op"] in ("rotate", "rotgrad"):
        n = (len(_rows(c)[0]) if c["hi"] > 1 else c["B"]) * (H + kv) * hd
        return {"bytes": n * (2 * e if c["op"] == "rotate" else e + 8), "flops": n * (8 if c["op"] == "rotate" else 16)}
    n = len(_rows(c)[0])
    return {"bytes": 2 * n * (row + kv * hd * e + 4), "flops": 2 * n * kv * hd}


# ---------------------------------------------------------------- the definitions in 64 bits

def _value(pool, e, page, off):
    """The rows (page, off) of a pool, [n, kv, head_dim], as the numbers they stand for."""
    at = pool.view(torch.uint8) if e is not None else pool
    x = at[page, :, off]
    if e is None:
        return x.double()
    return x.view(pool.dtype).double() * 2.0 ** (e[page, :, off].double() - 127.0)[..., None]


def _exact_attend(st):
    c = st["case"]
    out, lse = [], []
    for b, n in enumerate(_lengths(c)):
        j = torch.arange(n, device=st["q"].device)
        page = st["table"][b].long()[j // c["page"]] if n else j
        k, v = _value(st["k"], st["ke"], page, j % c["page"]), _value(st["v"], st["ve"], page, j % c["page"])
        far = float(n if c["pair"] else n - 1) - j.double()
        if c["pair"]:
            k, v = torch.cat((k, st["k_own"][b:b + 1].double())), torch.cat((v, st["v_own"][b:b + 1].double()))
            far = torch.cat((far, far.new_zeros(1)))
        if not len(k):
            out.append(k.new_zeros(c["heads"], c["hd"]))
            lse.append(k.new_full((c["heads"],), -math.inf))
            continue
        group = c["heads"] // c["kv"]
        k, v = (t.repeat_interleave(group, 1) for t in (k, v))                # [pairs, heads, head_dim]
        a = torch.einsum("hd,nhd->hn", st["q"][b].double(), k) * c["hd"] ** -0.5
        if st["slopes"] is not None:
            a = a - st["slopes"].double()[:, None] * far
        out.append(torch.einsum("hn,nhd->hd", torch.softmax(a, 1), v))
        lse.append(torch.logsumexp(a, 1))
    return torch.stack(out), torch.stack(lse)


def _exact_write(st):
    c = st["case"]
    pools, exps = [], []
    page, off = st["table"][st["seq"].long(), st["pos"].long() // c["page"]].long(), st["pos"].long() % c["page"]
    for rows, pool, e in ((st["k_rows"], st["k"], st["ke"]), (st["v_rows"], st["v"], st["ve"])):
        x = rows.double()
        new = pool.double()
        if e is not None:
            k = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 448.0)).clamp(min=-126.0)
            x = x / 2.0 ** k
            ex = 2.0 ** (e.double() - 127.0)
            ex[page, :, off] = 2.0 ** k[..., 0]
            exps.append(ex)
        new[page, :, off] = x
        pools.append(new)
    return tuple(pools + exps)


def _exact_rotate(st, grad=False):
    c = st["case"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=st["q"].device), st["pos"].double()[:, None] * st["freq"])[:, None, :]
    outs, ins, gains = [], [], []
    for n, g in (("q", "g_q"), ("k", "g_k")):
        x = st[n].detach().double().requires_grad_(grad)
        y = x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()
        if st[g] is not None:
            w = st[g].detach().double().requires_grad_(grad)
            gains.append(w)
            y = y * w.view(1, *x.shape[1:])
        part, rest = y.split([c["rot"], c["hd"] - c["rot"]], -1)
        if c["pairs"] == "halves":
            z = torch.complex(*part.chunk(2, -1)) * turn
            part = torch.cat((z.real, z.imag), -1)
        else:
            z = torch.complex(part[..., ::2], part[..., 1::2]) * turn
            part = torch.view_as_real(z).flatten(-2)
        ins.append(x)
        outs.append(torch.cat((part, rest), -1))
    if not grad:
        return tuple(outs)
    return torch.autograd.grad(outs, ins + gains, [st["dq_out"].double(), st["dk_out"].double()])


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(st)
    if case["op"] == "write":
        return _exact_write(st)
    if case["op"] == "read":
        at = st["table"][st["seq"].long(), st["pos"].long() // case["page"]].long(), st["pos"].long() % case["page"]
        return _value(st["k"], st["ke"], *at), _value(st["v"], st["ve"], *at)
    return _exact_rotate(st, case["op"] == "rotgrad")
