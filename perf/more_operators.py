"""The operators of a paged per-head KV cache held in 8 bits, over the sizes, types and options a serving program uses.

The cache's rows are e4m3 numbers with a power of two (an e8m0 number) per row: one token's keys, or values, of one KV
head. The exponent is the smallest with which the row's largest value is at most 448, and not below -110.

  paged_store_fp8      rows (a compressed cache's, say) to their slots, in 8 bits
  norm_rope_store_fp8  new tokens' queries, keys and values: per-head norm, rotation by position, the keys and values
                       to their slots, in 8 bits
  paged_attention_fp8  the new tokens' attention over the 8-bit rows of their segments, themselves included

Head counts are the repository's workloads' (28 query and 4 KV heads, 64 and 8, the tiny fp32 layer's 4 and 2 of
dimension 64). A case's lengths differ per head as the compression's budgets do.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
_EPS = 1e-6
_THETA = 1e6
_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


# ------------------------------------------------------------------ cases
def _attn(name, B, new, rows, *, ragged=False, hq=28, hkv=4, d=128, page=64, dtype="bf16", out=None, causal=True,
          lengths=1):
    """B sequences of `new` new tokens (ragged: 1 to new) over about `rows` earlier rows per KV head."""
    return dict(name=name, kind="attn", B=B, new=new, rows=rows, ragged=ragged, hq=hq, hkv=hkv, d=d, page=page,
                dtype=dtype, out=out or dtype, causal=causal, lengths=lengths)


def _rope(name, T, *, hq=28, hkv=4, d=128, rot=None, norm=True, pairs="halves", dtype="bf16", page=64, far=131072,
          factor=1.0):
    return dict(name=name, kind="rope", T=T, hq=hq, hkv=hkv, d=d, rot=d if rot is None else rot, norm=norm,
                pairs=pairs, dtype=dtype, page=page, far=far, factor=factor)


def _store(name, B, rows, *, hkv=4, d=128, page=64, dtype="bf16", lengths=1):
    return dict(name=name, kind="store", B=B, rows=rows, hkv=hkv, d=d, page=page, dtype=dtype, lengths=lengths)


def listed():
    return [
        # one generated token of one sequence over a compressed prompt: latency
        _attn("attn8_1x1_over_9k", 1, 1, 9000),
        # a generation step of a batch of long prompts, the throughput case
        _attn("attn8_40x1_over_30k", 40, 1, 30011),
        # drafted tokens being checked: 1 to 5 per sequence, 64 query and 8 KV heads
        _attn("attn8_16x5_over_25k", 16, 5, 25001, ragged=True, hq=64, hkv=8, page=32, out="f32"),
        # a follow-up question after the compression, of a length nobody chose
        _attn("attn8_1x1501_over_10k", 1, 1501, 10007),
        # long second turns of two sequences: the largest
        _attn("attn8_2x6000_over_20k", 2, 6000, 20480, hq=64, hkv=8, page=128),
        # the tiny fp32 layer of the end-to-end check, a short chunk each
        _attn("attn8_f32_5x37_over_900", 5, 37, 900, ragged=True, hq=4, hkv=2, d=64, page=16, dtype="f32"),
        # a generation step's 40 tokens, no norms (the models with 28 query heads have none)
        _rope("rope8_40", 40, norm=False),
        # a long chunk with norms of queries and keys, 64 query and 8 KV heads, positions to 256K
        _rope("rope8_6001_norm", 6001, hq=64, hkv=8, far=262144),
        # a chunk of fp32 rows, half of each head rotated in neighbouring pairs, positions scaled for a long context
        _rope("rope8_f32_1111_part", 1111, hq=16, hkv=8, d=64, rot=32, pairs="neighbours", dtype="f32", far=1 << 20,
              factor=1.25),
        # the rows of one tiny compressed fp32 layer
        _store("store8_tiny", 1, 512, hkv=2, d=64, page=16, dtype="f32"),
        # the rows of a batch of compressed 128K prompts
        _store("store8_8x32k", 8, 32768),
        # three prompts of an fp32 program, lengths that end inside a page
        _store("store8_f32_3x5001", 3, 5001, hkv=8, page=128, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ones' ranges: 1 to 64 sequences, 1 to 8192 new tokens over 1 to 64K rows, odd
    lengths among them, page sizes of 16 to 256 rows, both types, every head layout."""
    kind = rng.choice(("attn", "attn", "attn", "rope", "store"))
    hq, hkv, d = rng.choice([(28, 4, 128), (28, 4, 128), (64, 8, 128), (16, 2, 128), (8, 8, 64), (4, 2, 64),
                             (5, 1, 128)])
    page = rng.choice([16, 32, 64, 128, 256])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind == "attn":
        new = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 17, 8192)])
        rows = _log_int(rng, 1, 65536)
        B = _log_int(rng, 1, 64)
        # no more products than the largest listed case's, a sixteenth of that in fp32; 4 GB of rows at most
        pairs = 64 * 6000 * 2 * 23480 * 128 // (16 if dtype == "f32" else 1)
        while B > 1 and (B * hq * d * new * (rows + new / 2) > pairs or B * hkv * d * (rows + new) * 2 > 4 << 30):
            B -= 1
        if hq * d * new * (rows + new / 2) > pairs:
            new = max(1, int(pairs / (hq * d * (rows + new / 2))))
        case = _attn("", B, new, rows, ragged=rng.random() < 0.5, hq=hq, hkv=hkv, d=d, page=page, dtype=dtype,
                     out=rng.choice([dtype, "f32"]), causal=rng.random() < 0.85)
    elif kind == "rope":
        case = _rope("", min(_log_int(rng, 1, 8191), 6001 * 80 // (hq + 2 * hkv)), hq=hq, hkv=hkv, d=d,
                     rot=rng.choice([d, d, d // 2]), norm=rng.random() < 0.6,
                     pairs=rng.choice(["halves", "halves", "neighbours"]), dtype=dtype, page=page,
                     far=_log_int(rng, 1, 1 << 20), factor=rng.choice([1.0, 1.0, round(rng.uniform(1.0, 1.5), 3)]))
    else:
        case = _store("", _log_int(rng, 1, 8), _log_int(rng, 1, 32768), hkv=min(hkv, 4), d=d, page=page, dtype=dtype)
    if kind != "rope":
        case["lengths"] = rng.randrange(1 << 30)
    del case["name"]
    return case


# ------------------------------------------------------------------ lengths (host)
# A case's lengths are its own (drawn from case["lengths"]), the same for every seed.
def _head_shares(rng, hkv):
    """Shares of a layer's rows per KV head, mean 1, as head budgets come out: unequal by several times."""
    w = [0.25 + rng.betavariate(0.5, 2.0) for _ in range(hkv)]
    return [hkv * x / sum(w) for x in w]


def _near(rng, n):
    return 0 if n == 0 else max(1, int(n * rng.uniform(0.9, 1.1)))


def _lengths(case):
    """The case's lengths: per segment the rows before, per sequence the new tokens."""
    rng = random.Random(case["lengths"])
    hkv = case["hkv"]
    old, new = [], []
    for b in range(case["B"]):
        n = _near(rng, case["rows"])
        old += [int(n * f) for f in _head_shares(rng, hkv)]
        if case["kind"] == "attn":
            # the longest chunk is the first one, so that the bound a program passes is met
            new.append(rng.randint(1, case["new"]) if case["ragged"] and b else case["new"])
    return old, new


def _pages_of(rows, page):
    return [-(-r // page) for r in rows]


# ------------------------------------------------------------------ rows in 8 bits
def _quantise(x):
    """Rows [..., d] in fp32 or fp64 as e4m3 numbers and a power of two per row."""
    mantissa, exponent = torch.frexp(x.abs().amax(-1))
    e = torch.where(mantissa > 0.875, exponent - 8, exponent - 9).clamp(min=-110)
    scale = (e + 127).to(torch.uint8).view(_E8M0)
    return (x / scale.to(x.dtype).unsqueeze(-1)).float().to(_E4M3), scale


def _values(numbers, scales):
    return numbers.float() * scales.float().unsqueeze(-1)


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2654435761 % (1 << 62) + 4321)
    return g


def _randn(shape, g, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def _tables(counts, page_ids):
    """Tables whose rows hold consecutive pieces of page_ids; -1 past a segment's pages."""
    width = max(max(counts), 1)
    t = torch.full((len(counts), width), -1, dtype=torch.int32, device="cuda")
    used = torch.arange(width, device="cuda")[None, :] < torch.tensor(counts, device="cuda")[:, None]
    t[used] = page_ids[:sum(counts)].to(torch.int32)
    return t


def _channels(shape, g):
    """Sizes of a head's columns: most near 1, a few several times that, as the columns of keys come out."""
    c = torch.exp(0.3 * torch.randn(shape, generator=g, device="cuda"))
    return c * torch.where(torch.rand(shape, generator=g, device="cuda") < 0.04, 5.0, 1.0)


def _pool(n_pages, page, d, g):
    """A pool that other segments use too: rows of the model's sizes everywhere."""
    pool = {}
    for name in ("k", "v"):
        pool[name + "_pages"], pool[name + "_scales"] = _quantise(torch.randn((n_pages, page, d), generator=g,
                                                                              device="cuda"))
    return pool


def _prepare_attn(case, seed):
    g = _generator(seed)
    old, new = _lengths(case)
    hq, hkv, d, page, dt = case["hq"], case["hkv"], case["d"], case["page"], _DT[case["dtype"]]
    rows = [o + new[s // hkv] for s, o in enumerate(old)]
    counts = _pages_of(rows, page)
    n_pages = sum(counts) + 1 + sum(counts) // 16
    tables = _tables(counts, torch.randperm(n_pages, generator=g, device="cuda"))
    st = _pool(n_pages, page, d, g)
    # Every KV head has a direction that its queries share and its keys carry by a random amount, so that
    # logits spread as trained heads' do; a segment's first rows carry much of it (attention sinks).
    u = torch.randn((hkv, d), generator=g, device="cuda")
    dirs = u / u.norm(dim=-1, keepdim=True)
    sizes = _channels((hkv, d), g)
    for s in range(len(rows)):
        ids = tables[s, :counts[s]].long()
        c = torch.randn((len(ids), page, 1), generator=g, device="cuda")
        c[0, :4] = 3.0
        h = s % hkv
        k = _values(st["k_pages"][ids], st["k_scales"][ids]) * sizes[h] + 2.0 * c * dirs[h]
        numbers, scales = _quantise(k)
        st["k_pages"].view(torch.uint8)[ids] = numbers.view(torch.uint8)
        st["k_scales"].view(torch.uint8)[ids] = scales.view(torch.uint8)
    T = sum(new)
    q = torch.randn((T, hkv, hq // hkv, d), generator=g, device="cuda") / sizes[:, None, :]
    q = q + 1.25 * math.sqrt(d) * dirs[:, None, :]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    st.update(q=q.reshape(T, hq, d).to(dt), tables=tables, rows=_int32(rows), cu=_int32(cu), rows_host=rows,
              new_host=new, max_new=max(new))
    if own:
        import paper_2609_03235_amd as sg
        size = sg.paged_attention_fp8_workspace_size(st["q"], hkv, len(new), max_new=st["max_new"])
        st["workspace"] = sg.alloc_workspace(size, "cuda")
    return st


def _inv_freq(case):
    rot = case["rot"]
    f = _THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return (f / (4.0 if case["factor"] != 1.0 else 1.0)).float().cuda()  # scaled: positions four times as far


def _prepare_rope(case, seed):
    g = _generator(seed)
    T, hq, hkv, d, page, dt = case["T"], case["hq"], case["hkv"], case["d"], case["page"], _DT[case["dtype"]]
    sizes = torch.cat([torch.ones(hq * d, device="cuda"), _channels((hkv * d,), g),
                       torch.ones(hkv * d, device="cuda")])
    qkv = (torch.randn((T, (hq + 2 * hkv) * d), generator=g, device="cuda") * sizes).to(dt)  # one projection's output
    n_pages = -(-T * hkv // page) + 2
    slots = torch.randperm(n_pages * page, generator=g, device="cuda")[:T * hkv].to(torch.int32).reshape(T, hkv)
    if T > 8:
        slots[-3:] = -1  # a padded batch: the last tokens belong to nobody
    first = torch.randint(0, case["far"], (1,), generator=g, device="cuda")
    step = torch.randint(0, 2, (T,), generator=g, device="cuda")
    pos = (first + torch.arange(T, device="cuda") + 977 * step.cumsum(0) // 8).to(torch.int32)
    q, k, v = qkv.split([hq * d, hkv * d, hkv * d], dim=-1)
    w = [(1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dt) if case["norm"] else None for _ in range(2)]
    return dict(q=q.view(T, hq, d), k=k.view(T, hkv, d), v=v.view(T, hkv, d), positions=pos, slots=slots,
                inv_freq=_inv_freq(case), q_weight=w[0], k_weight=w[1], **_pool(n_pages, page, d, g))


def _prepare_store(case, seed):
    g = _generator(seed)
    rows, _ = _lengths(case)
    page, d, dt = case["page"], case["d"], _DT[case["dtype"]]
    counts = _pages_of(rows, page)
    n_pages = sum(counts) + 3
    tables = _tables(counts, torch.randperm(n_pages, generator=g, device="cuda"))
    N = sum(rows)
    seg = torch.repeat_interleave(torch.arange(len(rows)), torch.tensor(rows)).cuda()
    start = torch.tensor([0] + rows[:-1]).cumsum(0).cuda()
    at = torch.arange(N, device="cuda") - start[seg]
    slots = tables[seg, at // page] * page + (at % page).to(torch.int32)
    sizes = _channels((d,), g)
    return dict(k=(torch.randn((N, d), generator=g, device="cuda") * sizes).to(dt), v=_randn((N, d), g, dt),
                slots=slots.to(torch.int32), **_pool(n_pages, page, d, g))


def prepare(case, seed):
    st = {"attn": _prepare_attn, "rope": _prepare_rope, "store": _prepare_store}[case["kind"]](case, seed)
    st["case"] = dict(case)
    return st


def _pool_of(st):
    return {k: st[k] for k in ("k_pages", "v_pages", "k_scales", "v_scales")}


# ------------------------------------------------------------------ the framework's calls
def _run_own(st):
    import paper_2609_03235_amd as sg
    case = st["case"]
    if case["kind"] == "attn":
        out, lse = sg.paged_attention_fp8(st["q"], st["k_pages"], st["v_pages"], st["k_scales"], st["v_scales"],
                                          st["tables"], st["rows"], st["cu"], case["hkv"], max_new=st["max_new"],
                                          causal=case["causal"], out_dtype=_DT[case["out"]],
                                          workspace=st["workspace"])
        return dict(out=out, lse=lse)
    if case["kind"] == "rope":
        q = sg.norm_rope_store_fp8(st["q"], st["k"], st["v"], st["positions"], st["slots"], st["k_pages"],
                                   st["v_pages"], st["k_scales"], st["v_scales"], inv_freq=st["inv_freq"],
                                   q_weight=st["q_weight"], k_weight=st["k_weight"], eps=_EPS,
                                   interleaved=case["pairs"] == "neighbours", rope_factor=case["factor"])
        return dict(q=q, **_pool_of(st))
    sg.paged_store_fp8(st["k"], st["v"], st["slots"], st["k_pages"], st["v_pages"], st["k_scales"], st["v_scales"])
    return _pool_of(st)


# ------------------------------------------------------------------ plain forms
def _plain_attn(st):
    case = st["case"]
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    G, scale = hq // hkv, 1.0 / math.sqrt(d)
    q = st["q"]
    out = torch.empty(q.shape, dtype=_DT[case["out"]], device=q.device)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    rows = st["rows"].view(-1, hkv)
    t0 = 0
    for b, n in enumerate(st["new_host"]):
        # the heads' rows side by side, as many as the longest has; -1 in a table stands behind a head's last page
        L = max(st["rows_host"][b * hkv:(b + 1) * hkv])
        ids = st["tables"][b * hkv:(b + 1) * hkv, :-(-L // page)].long().clamp(min=0)
        k = _values(st["k_pages"][ids], st["k_scales"][ids]).view(hkv, -1, d)[:, :L]
        v = _values(st["v_pages"][ids], st["v_scales"][ids]).view(hkv, -1, d)[:, :L]
        kt = k.transpose(1, 2).contiguous()
        step = max(1, (1 << 28) // (hq * L))  # tokens whose logits are held at once
        for i in range(0, n, step):
            m = min(step, n - i)
            qs = q[t0 + i:t0 + i + m].float().view(m, hkv, G, d).transpose(0, 1).reshape(hkv, m * G, d)
            y = (torch.bmm(qs, kt) * scale).view(hkv, m, G, L)
            last = rows[b].view(hkv, 1) - 1
            if case["causal"]:
                last = last - n + 1 + i + torch.arange(m, device=q.device)
            else:
                last = last.expand(hkv, m)
            y = y.masked_fill(torch.arange(L, device=q.device) > last[:, :, None, None], -math.inf)
            top = y.amax(-1, keepdim=True)
            p = torch.exp(y - top)
            total = p.sum(-1, keepdim=True)
            o = torch.bmm(p.view(hkv, m * G, L), v).view(hkv, m, G, d) / total
            out[t0 + i:t0 + i + m] = o.transpose(0, 1).reshape(m, hq, d).to(out.dtype)
            lse[t0 + i:t0 + i + m] = (top + total.log()).squeeze(-1).transpose(0, 1).reshape(m, hq)
        t0 += n
    return dict(out=out, lse=lse)


def _plain_norm(x, w):
    x = x.float()
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * w.float()


def _plain_rotate(x, cos, sin, rot, pairs):
    y = x.clone()
    if pairs == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2] = a * cos - b * sin
        y[..., rot // 2:rot] = b * cos + a * sin
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2] = a * cos - b * sin
        y[..., 1:rot:2] = b * cos + a * sin
    return y


def _plain_put(pages, scales, slots, rows):
    """rows [N, d] into their slots; a slot of -1 keeps nothing."""
    keep = slots >= 0
    at = slots[keep].long()
    numbers, powers = _quantise(rows[keep])
    pages.view(torch.uint8).view(-1, pages.shape[-1])[at] = numbers.view(torch.uint8)
    scales.view(torch.uint8).view(-1)[at] = powers.view(torch.uint8)


def _plain_rope(st):
    case = st["case"]
    rot, dt = case["rot"], st["q"].dtype
    angle = st["positions"].double()[:, None, None] * st["inv_freq"].double()
    cos, sin = (angle.cos() * case["factor"]).float(), (angle.sin() * case["factor"]).float()
    q = _plain_rotate(_plain_norm(st["q"], st["q_weight"]), cos, sin, rot, case["pairs"]).to(dt)
    k = _plain_rotate(_plain_norm(st["k"], st["k_weight"]), cos, sin, rot, case["pairs"])
    slots = st["slots"].flatten()
    _plain_put(st["k_pages"], st["k_scales"], slots, k.flatten(0, 1))
    _plain_put(st["v_pages"], st["v_scales"], slots, st["v"].float().flatten(0, 1))
    return dict(q=q, **_pool_of(st))


def _plain_store(st):
    _plain_put(st["k_pages"], st["k_scales"], st["slots"], st["k"].float())
    _plain_put(st["v_pages"], st["v_scales"], st["slots"], st["v"].float())
    return _pool_of(st)


def run(state):
    if own:
        return _run_own(state)
    return {"attn": _plain_attn, "rope": _plain_rope, "store": _plain_store}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] == "attn":
        old, new = _lengths(case)
        hq, hkv, d, e = case["hq"], case["hkv"], case["d"], _BYTES[case["dtype"]]
        T = sum(new)
        rows = pairs = 0
        for s, o in enumerate(old):
            n = new[s // hkv]
            rows += o + n
            pairs += n * o + (n * (n + 1) // 2 if case["causal"] else n * n)
        return {"bytes": rows * 2 * (d + 1) + T * hq * (d * (e + _BYTES[case["out"]]) + 4) + 4 * (rows // case["page"]),
                "flops": 4 * d * (hq // hkv) * pairs}
    d, e = case["d"], _BYTES[case["dtype"]]
    if case["kind"] == "rope":
        T, hq, hkv = case["T"], case["hq"], case["hkv"]
        return {"bytes": T * ((2 * hq + 2 * hkv) * d * e + 2 * hkv * (d + 1) + 4 + 4 * hkv),
                "flops": T * (hq + 2 * hkv) * d * (8 if case["norm"] else 4)}
    rows, _ = _lengths(case)
    return {"bytes": sum(rows) * (2 * d * e + 2 * (d + 1) + 4), "flops": 0}


# ------------------------------------------------------------------ 64-bit values
def _decoded(numbers, scales):
    """Values of e4m3 and e8m0 numbers from their bits: sign, four exponent bits (bias 7), three of mantissa."""
    bits = numbers.view(torch.uint8).long()
    exponent, mantissa = bits >> 3 & 15, (bits & 7).double()
    size = torch.where(exponent == 0, mantissa * 2.0 ** -9,
                       (1 + mantissa / 8) * torch.exp2(exponent.double() - 7))
    power = torch.exp2(scales.view(torch.uint8).double() - 127)
    return torch.where(bits > 127, -size, size) * power.unsqueeze(-1)


def _exact_attn(case, st):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    G, page = hq // hkv, case["page"]
    q = st["q"].double()
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    t0 = 0
    for b, n in enumerate(st["new_host"]):
        for h in range(hkv):
            s = b * hkv + h
            L = st["rows_host"][s]
            r = torch.arange(L, device="cuda")
            pg, at = st["tables"][s].long()[r // page], r % page
            keys = _decoded(st["k_pages"].view(torch.uint8)[pg, at], st["k_scales"].view(torch.uint8)[pg, at])
            values = _decoded(st["v_pages"].view(torch.uint8)[pg, at], st["v_scales"].view(torch.uint8)[pg, at])
            for g in range(G):
                for i in range(0, n, 2048):
                    rows = slice(t0 + i, t0 + min(n, i + 2048))
                    y = torch.mm(q[rows, h * G + g], keys.t().contiguous()) / math.sqrt(d)
                    if case["causal"]:
                        seen = (L - n + i + torch.arange(y.shape[0], device="cuda"))[:, None] >= r[None, :]
                        y = torch.where(seen, y, torch.full_like(y, -math.inf))
                    z = torch.logsumexp(y, dim=1)
                    lse[rows, h * G + g] = z
                    out[rows, h * G + g] = torch.mm(torch.exp(y - z[:, None]), values)
        t0 += n
    return dict(out=out, lse=lse)


def _exact_put(st, name, slots, rows):
    """The pool's numbers and powers of two, those of `slots` from rows [N, d] in 64 bits, not rounded."""
    numbers = _decoded(st[name + "_pages"], torch.full_like(st[name + "_scales"].view(torch.uint8), 127))
    scales = torch.exp2(st[name + "_scales"].view(torch.uint8).double() - 127)
    keep = slots >= 0
    e = torch.ceil(torch.log2(rows[keep].abs().amax(-1) / 448)).clamp(min=-110)
    # log2 may be off by a rounding next to a power of two
    e = torch.where(rows[keep].abs().amax(-1) <= 224 * torch.exp2(e), (e - 1).clamp(min=-110), e)
    e = torch.where(rows[keep].abs().amax(-1) > 448 * torch.exp2(e), e + 1, e)
    at = slots[keep].long()
    numbers.view(-1, numbers.shape[-1])[at] = rows[keep] / torch.exp2(e).unsqueeze(-1)
    scales.view(-1)[at] = torch.exp2(e)
    return {name + "_pages": numbers, name + "_scales": scales}


def _exact_rope(case, st):
    d, rot = case["d"], case["rot"]
    half = rot // 2
    freq = torch.ones(d, dtype=torch.float64, device="cuda")
    partner = torch.arange(d, device="cuda")
    sign = torch.zeros(d, dtype=torch.float64, device="cuda")
    f = st["inv_freq"].double()
    for i in range(half):
        a, b = (i, i + half) if case["pairs"] == "halves" else (2 * i, 2 * i + 1)
        partner[a], partner[b] = b, a
        sign[a], sign[b] = -1.0, 1.0
    freq[sign < 0] = f
    freq[sign > 0] = f
    t = st["positions"].double()[:, None] * freq[None, :]
    cos = torch.where(sign == 0, torch.ones_like(t), torch.cos(t) * case["factor"])[:, None, :]
    sin = (torch.sin(t) * sign * case["factor"])[:, None, :]

    def turned(x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + _EPS) * w.double()
        return x * cos + x[..., partner] * sin

    slots = st["slots"].flatten()
    return dict(q=turned(st["q"], st["q_weight"]),
                **_exact_put(st, "k", slots, turned(st["k"], st["k_weight"]).flatten(0, 1)),
                **_exact_put(st, "v", slots, st["v"].double().flatten(0, 1)))


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "attn":
        return _exact_attn(case, st)
    if case["kind"] == "rope":
        return _exact_rope(case, st)
    return dict(**_exact_put(st, "k", st["slots"], st["k"].double()),
                **_exact_put(st, "v", st["slots"], st["v"].double()))
