"""The operators of a paged per-head KV cache, over the sizes, types and options a serving program uses.

After a prompt's cache is compressed every KV head of every sequence (a segment) holds its own number
of rows. A serving program keeps the segments in pages of one pool and then works in steps of new tokens:

  page_update      pages taken from (or given back to) the free stack for the rows every segment gains
                   or loses, and the slot of every new row
  paged_store      rows (a compressed cache's, say) copied to their slots
  norm_rope_store  new tokens' queries, keys and values: per-head norm, rotation by position, the keys
                   and values to their slots
  paged_attention  the new tokens' attention over the rows of their segments, themselves included

Head counts are the repository's workloads' (28 query and 4 KV heads, 64 and 8, the tiny fp32 layer's
4 and 2 of dimension 64). A case's lengths differ per head as the compression's budgets do.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
_EPS = 1e-6
_THETA = 1e6


# ------------------------------------------------------------------ cases
def _attn(name, B, new, rows, *, ragged=False, hq=28, hkv=4, d=128, page=64, dtype="bf16", out=None, causal=True,
          lengths=1):
    """B sequences of `new` new tokens (ragged: 1 to new) over about `rows` earlier rows per KV head."""
    return dict(name=name, kind="attn", B=B, new=new, rows=rows, ragged=ragged, hq=hq, hkv=hkv, d=d, page=page,
                dtype=dtype, out=out or dtype, causal=causal, lengths=lengths)


def _rope(name, T, *, hq=28, hkv=4, d=128, rot=None, norm=True, pairs="halves", dtype="bf16", page=64, far=131072):
    return dict(name=name, kind="rope", T=T, hq=hq, hkv=hkv, d=d, rot=d if rot is None else rot, norm=norm,
                pairs=pairs, dtype=dtype, page=page, far=far)


def _pages(name, B, rows, add, *, hkv=4, page=64, order="token", drop=0, lengths=1):
    """B sequences with about `rows` rows per KV head: each gains up to `add` tokens (or, by segment, about
    `add` rows per head); every drop-th sequence gives rows back instead."""
    return dict(name=name, kind="pages", B=B, rows=rows, add=add, hkv=hkv, page=page, order=order, drop=drop,
                lengths=lengths)


def _store(name, B, rows, *, hkv=4, d=128, page=64, dtype="bf16", lengths=1):
    return dict(name=name, kind="store", B=B, rows=rows, hkv=hkv, d=d, page=page, dtype=dtype, lengths=lengths)


def listed():
    return [
        # one generated token of one sequence whose 32K prompt was compressed to a quarter: latency
        _attn("attn_1x1_over_8k", 1, 1, 8192),
        # a generation step of a batch of long prompts, the throughput case
        _attn("attn_32x1_over_32k", 32, 1, 32768),
        # drafted tokens being checked: 1 to 6 per sequence, 64 query and 8 KV heads
        _attn("attn_16x6_over_20k", 16, 6, 20011, ragged=True, hq=64, hkv=8, page=32, out="f32"),
        # a follow-up question after the compression, of a length nobody chose
        _attn("attn_1x1999_over_8k", 1, 1999, 8192),
        # long second turns of two sequences: the largest
        _attn("attn_2x8192_over_16k", 2, 8192, 16384, hq=64, hkv=8, page=128),
        # the tiny fp32 layer of the end-to-end check, a short chunk each
        _attn("attn_f32_3x50_over_1k", 3, 50, 1000, ragged=True, hq=4, hkv=2, d=64, page=16, dtype="f32"),
        # a generation step's 32 tokens, no norms (the models with 28 query heads have none)
        _rope("rope_32", 32, norm=False),
        # a long chunk with norms of queries and keys, 64 query and 8 KV heads, positions to 256K
        _rope("rope_8191_norm", 8191, hq=64, hkv=8, far=262144),
        # one more token for each of 64 sequences, a few of which just finished and give their pages back
        _pages("pages_64x1", 64, 5000, 1, hkv=8, page=16, drop=13),
        # the pages and slots of 16 compressed prompts
        _pages("pages_16_prompts", 16, 0, 32768, page=64, order="segment"),
        # the rows of one tiny compressed fp32 layer
        _store("store_tiny", 1, 512, hkv=2, d=64, page=16, dtype="f32"),
        # the rows of a batch of compressed 128K prompts
        _store("store_8x32k", 8, 32768),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ones' ranges: 1 to 64 sequences, 1 to 8192 new tokens over 1 to 64K rows, odd
    lengths among them, page sizes of 16 to 256 rows, both types, every head layout."""
    kind = rng.choice(("attn", "attn", "attn", "rope", "rope", "pages", "store"))
    hq, hkv, d = rng.choice([(28, 4, 128), (28, 4, 128), (64, 8, 128), (16, 2, 128), (8, 8, 64), (4, 2, 64),
                             (5, 1, 128)])
    page = rng.choice([16, 32, 64, 128, 256])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind == "attn":
        new = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 17, 8192)])
        rows = _log_int(rng, 1, 65536)
        B = _log_int(rng, 1, 64)
        # no more products than the largest listed case's, a sixteenth of that in fp32; 8 GB of rows at most
        pairs = 64 * 8192 * 2 * 20480 * 128 // (16 if dtype == "f32" else 1)
        while B > 1 and (B * hq * d * new * (rows + new / 2) > pairs or B * hkv * d * (rows + new) * 4 > 4 << 30):
            B -= 1
        if hq * d * new * (rows + new / 2) > pairs:
            new = max(1, int(pairs / (hq * d * (rows + new / 2))))
        case = _attn("", B, new, rows, ragged=rng.random() < 0.5, hq=hq, hkv=hkv, d=d, page=page, dtype=dtype,
                     out=rng.choice([dtype, "f32"]), causal=rng.random() < 0.85)
    elif kind == "rope":
        case = _rope("", min(_log_int(rng, 1, 8191), 8191 * 72 // (hq + 2 * hkv)), hq=hq, hkv=hkv, d=d,
                     rot=rng.choice([d, d, d // 2]), norm=rng.random() < 0.6,
                     pairs=rng.choice(["halves", "halves", "neighbours"]), dtype=dtype, page=page,
                     far=_log_int(rng, 1, 1 << 20))
    elif kind == "pages":
        if rng.random() < 0.5:
            case = _pages("", _log_int(rng, 1, 64), rng.choice([0, _log_int(rng, 1, 20000)]), _log_int(rng, 1, 2048),
                          hkv=hkv, page=page, drop=rng.choice([0, 3, 13]))
        else:
            case = _pages("", _log_int(rng, 1, 16), rng.choice([0, _log_int(rng, 1, 5000)]), _log_int(rng, 1, 32768),
                          hkv=hkv, page=page, order="segment", drop=rng.choice([0, 0, 5]))
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
    """The case's lengths: per sequence the new tokens, per segment the rows before."""
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


def _page_lengths(case):
    rng = random.Random(case["lengths"])
    hkv, B = case["hkv"], case["B"]
    old, add = [], []
    for b in range(B):
        n = _near(rng, case["rows"])
        mine = [int(n * f) for f in _head_shares(rng, hkv)]
        old += mine
        drop = case["drop"] and b % case["drop"] == case["drop"] - 1
        if case["order"] == "token":
            add.append(-rng.choice([1, 7, n + 50000]) if drop else rng.randint(1, case["add"]))
        elif drop:
            add += [-rng.randint(0, m) for m in mine]
        else:
            m = _near(rng, case["add"])
            add += [int(m * f) for f in _head_shares(rng, hkv)]
    return old, add


def _store_rows(case):
    rng = random.Random(case["lengths"])
    rows = []
    for _ in range(case["B"]):
        n = _near(rng, case["rows"])
        rows += [int(n * f) for f in _head_shares(rng, case["hkv"])]
    return rows


def _pages_of(rows, page):
    return [-(-r // page) for r in rows]


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


def _prepare_attn(case, seed):
    g = _generator(seed)
    old, new = _lengths(case)
    hq, hkv, d, page, dt = case["hq"], case["hkv"], case["d"], case["page"], _DT[case["dtype"]]
    rows = [o + new[s // hkv] for s, o in enumerate(old)]
    counts = _pages_of(rows, page)
    n_pages = sum(counts) + 1 + sum(counts) // 16
    tables = _tables(counts, torch.randperm(n_pages, generator=g, device="cuda"))
    # Every KV head has a direction that its queries share and its keys carry by a random amount, so that
    # logits spread as trained heads' do; a segment's first rows carry much of it (attention sinks).
    u = torch.randn((hkv, d), generator=g, device="cuda")
    k_pages = _randn((n_pages, page, d), g, dt)
    v_pages = _randn((n_pages, page, d), g, dt)
    dirs = u / u.norm(dim=-1, keepdim=True)
    for s in range(len(rows)):
        ids = tables[s, :counts[s]].long()
        c = torch.randn((len(ids), page, 1), generator=g, device="cuda")
        c[0, :4] = 3.0
        k_pages[ids] = (k_pages[ids].float() + 2.0 * c * dirs[s % hkv]).to(dt)
    T = sum(new)
    q = torch.randn((T, hkv, hq // hkv, d), generator=g, device="cuda") + 1.25 * math.sqrt(d) * dirs[:, None, :]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    st = dict(q=q.reshape(T, hq, d).to(dt), k_pages=k_pages, v_pages=v_pages, tables=tables, rows=_int32(rows),
              cu=_int32(cu), rows_host=rows, new_host=new, max_new=max(new))
    if own:
        import paper_2609_03235_amd as sg
        size = sg.paged_attention_workspace_size(st["q"], case["hkv"], len(new), max_new=st["max_new"])
        st["workspace"] = sg.alloc_workspace(size, "cuda")
    return st


def _inv_freq(rot):
    return (_THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()


def _prepare_rope(case, seed):
    g = _generator(seed)
    T, hq, hkv, d, page, dt = case["T"], case["hq"], case["hkv"], case["d"], case["page"], _DT[case["dtype"]]
    qkv = _randn((T, (hq + 2 * hkv) * d), g, dt)  # one fused projection's output
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
                k_pages=_randn((n_pages, page, d), g, dt), v_pages=_randn((n_pages, page, d), g, dt),
                inv_freq=_inv_freq(case["rot"]), q_weight=w[0], k_weight=w[1])


def _prepare_pages(case, seed):
    g = _generator(seed)
    old, add = _page_lengths(case)
    hkv, page = case["hkv"], case["page"]
    by_token = case["order"] == "token"
    per_seg = [add[s // hkv] if by_token else add[s] for s in range(len(old))]
    counts = _pages_of(old, page)
    after = _pages_of([max(0, o + a) for o, a in zip(old, per_seg)], page)
    n_pages = sum(counts) + sum(after) + 7
    perm = torch.randperm(n_pages, generator=g, device="cuda")
    width = max(max(counts), max(after)) + 3
    tables = torch.full((len(old), width), -1, dtype=torch.int32, device="cuda")
    tables[:, :max(max(counts), 1)] = _tables(counts, perm)
    # the stack: entries below the head were handed out, those from it on are free
    head = sum(counts)
    gains = sum(max(a, 0) for a in add)
    return dict(rows=_int32(old), add=_int32(add), tables=tables, free_pages=perm.to(torch.int32), head=_int32([head]),
                n_slots=gains + (5 if by_token else 0))  # a padded batch has a few tokens more


def _prepare_store(case, seed):
    g = _generator(seed)
    rows = _store_rows(case)
    page, d, dt = case["page"], case["d"], _DT[case["dtype"]]
    counts = _pages_of(rows, page)
    n_pages = sum(counts) + 3
    tables = _tables(counts, torch.randperm(n_pages, generator=g, device="cuda"))
    N = sum(rows)
    seg = torch.repeat_interleave(torch.arange(len(rows)), torch.tensor(rows)).cuda()
    start = torch.tensor([0] + rows[:-1]).cumsum(0).cuda()
    at = torch.arange(N, device="cuda") - start[seg]
    slots = tables[seg, at // page] * page + (at % page).to(torch.int32)
    return dict(k=_randn((N, d), g, dt), v=_randn((N, d), g, dt), slots=slots.to(torch.int32),
                k_pages=_randn((n_pages, page, d), g, dt), v_pages=_randn((n_pages, page, d), g, dt))


def prepare(case, seed):
    st = {"attn": _prepare_attn, "rope": _prepare_rope, "pages": _prepare_pages,
          "store": _prepare_store}[case["kind"]](case, seed)
    st["case"] = dict(case)
    return st


# ------------------------------------------------------------------ the framework's calls
def _run_own(st):
    import paper_2609_03235_amd as sg
    case = st["case"]
    if case["kind"] == "attn":
        out, lse = sg.paged_attention(st["q"], st["k_pages"], st["v_pages"], st["tables"], st["rows"], st["cu"],
                                      case["hkv"], max_new=st["max_new"], causal=case["causal"],
                                      out_dtype=_DT[case["out"]], workspace=st["workspace"])
        return dict(out=out, lse=lse)
    if case["kind"] == "rope":
        q = sg.norm_rope_store(st["q"], st["k"], st["v"], st["positions"], st["slots"], st["k_pages"], st["v_pages"],
                               inv_freq=st["inv_freq"], q_weight=st["q_weight"], k_weight=st["k_weight"], eps=_EPS,
                               interleaved=case["pairs"] == "neighbours")
        return dict(q=q, k_pages=st["k_pages"], v_pages=st["v_pages"])
    if case["kind"] == "pages":
        return sg.page_update(st["rows"], st["add"], st["tables"], st["free_pages"], st["head"],
                              page_size=case["page"], n_slots=st["n_slots"], by_segment=case["order"] == "segment")
    sg.paged_store(st["k"], st["v"], st["slots"], st["k_pages"], st["v_pages"])
    return dict(k_pages=st["k_pages"], v_pages=st["v_pages"])


# ------------------------------------------------------------------ plain forms
def _segment_rows(st, s, n):
    """The n rows of segment s, keys and values, as they lie in the pool."""
    page = st["k_pages"].shape[1]
    ids = st["tables"][s, :-(-n // page)].long()
    return st["k_pages"][ids].flatten(0, 1)[:n], st["v_pages"][ids].flatten(0, 1)[:n]


def _plain_attn(st):
    case = st["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    G, scale = hq // hkv, 1.0 / math.sqrt(d)
    q = st["q"]
    out = torch.empty(q.shape, dtype=_DT[case["out"]], device=q.device)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    t0 = 0
    for b, n in enumerate(st["new_host"]):
        for h in range(hkv):
            L = st["rows_host"][b * hkv + h]
            k, v = (x.float() for x in _segment_rows(st, b * hkv + h, L))
            step = max(1, (1 << 28) // (G * L))  # tokens whose logits are held at once
            for i in range(0, n, step):
                m = min(step, n - i)
                qs = q[t0 + i:t0 + i + m, h * G:(h + 1) * G].float().reshape(m * G, d)
                y = (qs @ k.T * scale).view(m, G, L)
                if case["causal"]:
                    last = L - n + i + torch.arange(m, device=q.device)
                    y = y.masked_fill(torch.arange(L, device=q.device) > last[:, None, None], -math.inf)
                top = y.amax(-1, keepdim=True)
                p = torch.exp(y - top)
                total = p.sum(-1, keepdim=True)
                o = (p.view(m * G, L) @ v).view(m, G, d) / total
                out[t0 + i:t0 + i + m, h * G:(h + 1) * G] = o.to(out.dtype)
                lse[t0 + i:t0 + i + m, h * G:(h + 1) * G] = (top + total.log()).squeeze(-1)
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


def _plain_put(pages, slots, rows):
    """rows [N, d] into their slots; a slot of -1 keeps nothing."""
    flat = pages.view(-1, pages.shape[-1])
    keep = slots >= 0
    flat[slots[keep].long()] = rows[keep].to(pages.dtype)


def _plain_rope(st):
    case = st["case"]
    rot, dt = case["rot"], st["q"].dtype
    angle = st["positions"].double()[:, None, None] * st["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _plain_rotate(_plain_norm(st["q"], st["q_weight"]), cos, sin, rot, case["pairs"]).to(dt)
    k = _plain_rotate(_plain_norm(st["k"], st["k_weight"]), cos, sin, rot, case["pairs"])
    slots = st["slots"].flatten()
    _plain_put(st["k_pages"], slots, k.flatten(0, 1))
    _plain_put(st["v_pages"], slots, st["v"].flatten(0, 1))
    return dict(q=q, k_pages=st["k_pages"], v_pages=st["v_pages"])


def _plain_pages(st):
    case = st["case"]
    P, hkv, n_slots = case["page"], case["hkv"], st["n_slots"]
    rows, tables, free = st["rows"].long(), st["tables"], st["free_pages"]
    S, width = tables.shape
    add = st["add"].long()
    gain = add.clamp(min=0)
    per_seg = add if case["order"] == "segment" else add.repeat_interleave(hkv, output_size=S)
    after = (rows + per_seg).clamp(min=0)
    p0, p1 = (rows + P - 1) // P, (after + P - 1) // P
    taken, given = (p1 - p0).clamp(min=0), (p0 - p1).clamp(min=0)
    head = st["head"].long()
    base = head - given.sum()
    j = torch.arange(width, device=rows.device)[None, :]
    # given back: pages [p1, p0) of each segment in order, onto the stack below its head
    back = (j >= p1[:, None]) & (j < p0[:, None])
    where = base + (given.cumsum(0) - given)[:, None] + j - p1[:, None]
    spare = torch.cat([free, free.new_zeros(1)])
    spare.scatter_(0, torch.where(back, where, free.numel()).flatten(), tables.flatten())
    free.copy_(spare[:-1])
    # taken: off the stack in segment order
    take = (j >= p0[:, None]) & (j < p1[:, None])
    src = (base + (taken.cumsum(0) - taken)[:, None] + j - p0[:, None]).clamp(0, free.numel() - 1)
    tables.copy_(torch.where(take, free[src], tables))
    cu = torch.cat([gain.new_zeros(1), gain.cumsum(0)])
    i = torch.arange(n_slots, device=rows.device)
    owner = torch.searchsorted(cu, i, right=True) - 1
    real = i < cu[-1]
    owner = owner.clamp(max=gain.numel() - 1)
    if case["order"] == "segment":
        at = rows[owner] + i - cu[owner]
        slots = tables[owner, (at // P).clamp(max=width - 1)].long() * P + at % P
        slots = torch.where(real, slots, -1)
    else:
        seg = owner[:, None] * hkv + torch.arange(hkv, device=rows.device)
        at = rows[seg] + (i - cu[owner])[:, None]
        slots = tables[seg, (at // P).clamp(max=width - 1)].long() * P + at % P
        slots = torch.where(real[:, None], slots, -1)
    return dict(slots=slots.to(torch.int32), rows=after.to(torch.int32), head=(base + taken.sum()).to(torch.int32),
                cu=cu.to(torch.int32), status=torch.zeros(1, dtype=torch.int32, device=rows.device), tables=tables,
                free_pages=free)


def _plain_store(st):
    _plain_put(st["k_pages"], st["slots"], st["k"])
    _plain_put(st["v_pages"], st["slots"], st["v"])
    return dict(k_pages=st["k_pages"], v_pages=st["v_pages"])


def run(state):
    if own:
        return _run_own(state)
    return {"attn": _plain_attn, "rope": _plain_rope, "pages": _plain_pages,
            "store": _plain_store}[state["case"]["kind"]](state)


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
        return {"bytes": rows * 2 * d * e + T * hq * (d * (e + _BYTES[case["out"]]) + 4) + 4 * (rows // case["page"]),
                "flops": 4 * d * (hq // hkv) * pairs}
    if case["kind"] == "rope":
        heads = case["hq"] + 2 * case["hkv"]
        n, e = case["T"] * heads * case["d"], _BYTES[case["dtype"]]
        return {"bytes": 2 * n * e + case["T"] * (4 + 4 * case["hkv"]), "flops": n * (8 if case["norm"] else 4)}
    if case["kind"] == "pages":
        old, add = _page_lengths(case)
        S, per_token = len(old), case["hkv"] if case["order"] == "token" else 1
        gains = sum(max(a, 0) for a in add)
        if case["order"] == "token":
            add = [add[s // case["hkv"]] for s in range(S)]
        moved = sum(abs(a - b) for a, b in zip(_pages_of([max(0, o + x) for o, x in zip(old, add)], case["page"]),
                                               _pages_of(old, case["page"])))
        return {"bytes": 4 * (gains * per_token + 4 * S + 2 * moved), "flops": 0}
    return {"bytes": sum(_store_rows(case)) * (4 * case["d"] * _BYTES[case["dtype"]] + 4), "flops": 0}


# ------------------------------------------------------------------ 64-bit values
def _exact_attn(case, st):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    G, page = hq // hkv, case["page"]
    q = st["q"].double()
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    kf = st["k_pages"].view(-1, d)
    vf = st["v_pages"].view(-1, d)
    t0 = 0
    for b, n in enumerate(st["new_host"]):
        for h in range(hkv):
            s = b * hkv + h
            L = st["rows_host"][s]
            r = torch.arange(L, device="cuda")
            slot = st["tables"][s].long()[r // page] * page + r % page
            keys, values = kf[slot].double(), vf[slot].double()
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
    first = sign < 0
    second = sign > 0
    freq[first] = f
    freq[second] = f
    t = st["positions"].double()[:, None] * freq[None, :]
    cos = torch.where(sign == 0, torch.ones_like(t), torch.cos(t))[:, None, :]
    sin = (torch.sin(t) * sign)[:, None, :]

    def turned(x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + _EPS) * w.double()
        return x * cos + x[..., partner] * sin

    k_pages, v_pages = st["k_pages"].double(), st["v_pages"].double()
    slots = st["slots"].long()
    k = turned(st["k"], st["k_weight"])
    for h in range(case["hkv"]):
        ok = slots[:, h] >= 0
        k_pages.view(-1, d)[slots[ok, h]] = k[ok, h]
        v_pages.view(-1, d)[slots[ok, h]] = st["v"][ok, h].double()
    return dict(q=turned(st["q"], st["q_weight"]), k_pages=k_pages, v_pages=v_pages)


def exact(case, seed):
    if case["kind"] == "attn":
        return _exact_attn(case, prepare(case, seed))
    if case["kind"] == "rope":
        return _exact_rope(case, prepare(case, seed))
    if case["kind"] == "store":
        st = prepare(case, seed)
        k_pages, v_pages = st["k_pages"].double(), st["v_pages"].double()
        k_pages.view(-1, case["d"])[st["slots"].long()] = st["k"].double()
        v_pages.view(-1, case["d"])[st["slots"].long()] = st["v"].double()
        return dict(k_pages=k_pages, v_pages=v_pages)
    return None  # whole numbers
