"""The paged per-head cache on an MI355X: pages and slots, rows into pages, norm and rotation, attention
of new tokens, each against a plain implementation in 64 bits (or in whole numbers).

Tolerances of the attention, derived before the first run. With y the logits, A = sum p |v| / sum p:
  * a logit is the fp32 sum of exact products (bf16) or of fp32 ones, off by at most
    delta = 2^-21 scale max_r sum_d |q_d k_d| (DELTA below also holds the rounding of the exponent's
    fp32 argument and of exp2, 2^-22 (1 + |y|)); a weight is then off by 2 delta relative;
  * probabilities are rounded to bf16 (half a step: 2^-8 relative) for bf16 output of bf16 inputs, or keep
    their fp32 bits (2^-24), as they do for bf16 output too up to 48 query rows per KV head;
  * an fp32 accumulator takes one rounding per 16 keys and one per merged part: (rows / 4 + 64) 2^-24 A
    covers them at four roundings each;
  * the output is rounded to its type: half a step of |o|.
The log-sum-exp is off by delta + 2^-21 (1 + |lse|) at most.
"""
import math

import pytest
import torch

import paper_2609_03235_amd as sg

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def _say(msg):
    print(f"[gpu case] {msg}", flush=True)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------ pages and slots
def _plain_update(rows, add, tables, free, head, page, n_slots, hkv, by_segment):
    """page_update with lists of Python integers."""
    rows, tables, free = list(rows), [list(t) for t in tables], list(free)
    S = len(rows)
    width = len(tables[0])
    per_seg = [add[s] if by_segment else add[s // hkv] for s in range(S)]
    after = [max(0, r + a) for r, a in zip(rows, per_seg)]
    pages = lambda r: -(-r // page)
    gains = [max(a, 0) for a in add]
    given = [p for s in range(S) for p in tables[s][pages(after[s]):pages(rows[s])]]
    taken = sum(max(0, pages(after[s]) - pages(rows[s])) for s in range(S))
    base = head - len(given)
    status = 0
    if any(not 0 <= r <= width * page or a > width * page for r, a in zip(rows, after)):
        status = 2
    elif not 0 <= head <= len(free) or base < 0:
        status = 3
    elif sum(gains) > n_slots:
        status = 4
    elif base + taken > len(free):
        status = 1
    items = n_slots if by_segment else n_slots * hkv
    if status:
        return dict(slots=[-1] * items, rows=rows, head=head, cu=[0] * (len(add) + 1), status=status, tables=tables,
                    free_pages=free)
    free[base:head] = given
    at = base
    for s in range(S):
        for j in range(pages(rows[s]), pages(after[s])):
            tables[s][j] = free[at]
            at += 1
    slot = lambda s, p: tables[s][p // page] * page + p % page
    slots, cu = [], [0]
    for i, g in enumerate(gains):
        for t in range(g):
            slots += [slot(i, rows[i] + t)] if by_segment else \
                [slot(i * hkv + h, rows[i * hkv + h] + t) for h in range(hkv)]
        cu.append(cu[-1] + g)
    return dict(slots=slots + [-1] * (items - len(slots)), rows=after, head=at, cu=cu, status=0, tables=tables,
                free_pages=free)


def _start(rows, page, width, n_pages, seed):
    """Tables of pages handed out in a random order, and the stack behind them."""
    g = torch.Generator().manual_seed(seed)
    perm = torch.randperm(n_pages, generator=g).tolist()
    tables, head = [], 0
    for r in rows:
        n = -(-r // page)
        tables.append(perm[head:head + n] + [-1] * (width - n))
        head += n
    return tables, perm, head


def _update_both(rows, add, tables, free, head, page, n_slots, hkv, by_segment, **kw):
    want = _plain_update(rows, add, tables, free, head, page, n_slots, hkv, by_segment)
    got = sg.page_update(_i32(rows), _i32(add), _i32(tables), _i32(free), _i32([head]), page_size=page,
                         n_slots=n_slots, by_segment=by_segment, **kw)
    _check_update(got, want)
    return got, want


def _check_update(got, want):
    for name, w in want.items():
        g = got[name].flatten().tolist()
        w = [x for t in w for x in t] if name == "tables" else (w if isinstance(w, list) else [w])
        assert g == w, (name, g[:20], w[:20])


PAGE_CASES = [
    # rows, add, hkv, page, by_segment, spare slots
    ([0], [1], 1, 16, False, 0),
    ([15, 16, 17, 0], [1, 1], 2, 16, False, 3),
    ([15, 16, 17, 0], [0, -5], 2, 16, False, 2),
    ([100, 7, 33, 64], [-100, 40], 2, 32, False, 0),
    ([100, 7, 33, 64], [-1000, 200, 0, -32], 1, 16, True, 5),
    ([0] * 6, [5000, 1, 0, 777, 16, 17], 1, 64, True, 0),
    ([5] * 64, [i % 7 - 2 for i in range(32)], 2, 16, False, 9),
    ([300] * 600, [(i * 37) % 90 - 30 for i in range(200)], 3, 16, False, 0),
    ([13] * 2048, [(i * 97) % 50 for i in range(2048)], 1, 16, True, 1),
    ([0] * 8, [20011, 9999, 31111, 1, 0, 44444, 5, 12345], 1, 128, True, 7),
    ([60000, 3, 60000, 9], [-60000, 50000], 2, 16, False, 0),  # given back and taken in one call, many workgroups
]


@pytest.mark.parametrize("rows,add,hkv,page,by_segment,spare", PAGE_CASES)
def test_page_update(rows, add, hkv, page, by_segment, spare):
    _say(f"page_update {len(rows)} segments, {len(add)} adds, page {page}")
    gains = sum(max(a, 0) for a in add)
    most = max(r + max(a, 0) for r in rows for a in add)
    tables, free, head = _start(rows, page, -(-most // page) + 2, sum(-(-(r + most) // page) for r in rows) + 5, 3)
    _update_both(rows, add, tables, free, head, page, gains + spare, hkv, by_segment)


def test_page_update_failures_change_nothing():
    _say("page_update failures")
    rows, page = [40, 40, 10, 0], 16
    tables, free, head = _start(rows, page, 5, 9, 1)
    for add, n_slots, head_, seg in [([10, 30], 64, head, False), ([41, 0], 64, head, False), ([1, 1], 1, head, False),
                                     ([1, 1], 2, 10, False), ([1, 1], 2, -1, False), ([-40, 1], 2, 2, False),
                                     ([0, 0, 0, 33], 64, head, True)]:
        got, want = _update_both(rows, add, tables, free, head_, page, n_slots, 1 if seg else 2, seg)
        assert want["status"] != 0
    bad_rows = [40, -1, 10, 0]
    _, want = _update_both(bad_rows, [1, 1], tables, free, head, page, 2, 2, False)
    assert want["status"] == 2


@pytest.mark.parametrize("n", [1, 60000])
def test_page_update_in_place(n):
    """rows and head updated in place, in one workgroup and with many; two calls in a row."""
    _say(f"page_update in place {n}")
    page, hkv = 16, 2
    rows = [33, 50, 0, 7]
    tables, free, head = _start(rows, page, (n * 2 + 64) // page + 1, n // 2 + 200, 5)
    tables = [t + [-1] * (2 * n // page + 8) for t in tables]
    free = free + list(range(len(free), len(free) + n))
    d = dict(rows=_i32(rows), tables=_i32(tables), free=_i32(free), head=_i32([head]))
    state = (rows, tables, free, head)
    for add in ([n, 1], [-7, n]):
        want = _plain_update(state[0], add, state[1], state[2], state[3], page, n + 1, hkv, False)
        got = sg.page_update(d["rows"], _i32(add), d["tables"], d["free"], d["head"], page_size=page, n_slots=n + 1,
                             rows_out=d["rows"], head_out=d["head"])
        _check_update(got, want)
        state = (want["rows"], want["tables"], want["free_pages"], want["head"])


# ------------------------------------------------------------------ rows into pages
@pytest.mark.parametrize("dtype,d,n,page", [(BF, 128, 1, 16), (BF, 64, 777, 16), (F32, 128, 1000, 64), (F32, 64, 3, 32),
                                            (BF, 128, 20001, 256)])
def test_paged_store(dtype, d, n, page):
    _say(f"paged_store {n} rows of {d}")
    g = torch.Generator(device=DEV).manual_seed(n)
    pages = -(-n // page) + 3
    k, v = (torch.randn(n, d, generator=g, device=DEV).to(dtype) for _ in range(2))
    kp, vp = (torch.randn(pages, page, d, generator=g, device=DEV).to(dtype) for _ in range(2))
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:n].to(torch.int32)
    slots[::5] = -1
    if n > 3:
        slots[3] = pages * page  # just past the pool
        slots[2] = 2**31 - 1
    wk, wv = kp.clone(), vp.clone()
    ok = (slots >= 0) & (slots < pages * page)
    wk.view(-1, d)[slots[ok].long()] = k[ok]
    wv.view(-1, d)[slots[ok].long()] = v[ok]
    sg.paged_store(k, v, slots, kp, vp)
    assert torch.equal(kp, wk) and torch.equal(vp, wv)


def test_paged_store_of_nothing():
    kp = torch.zeros(1, 16, 64, device=DEV)
    sg.paged_store(kp[:0, 0], kp[:0, 0], _i32([]), kp, kp.clone())
    assert not kp.any()


# ------------------------------------------------------------------ norm and rotation
def _plain_rope(x, w, pos, inv_freq, eps, interleaved):
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    if inv_freq is None:
        return x
    half = inv_freq.numel()
    t = pos.double()[:, None] * inv_freq.double()
    cos, sin = torch.cos(t)[:, None], torch.sin(t)[:, None]
    y = x.clone()
    ia = torch.arange(half, device=x.device) * (2 if interleaved else 1)
    ib = ia + (1 if interleaved else half)
    y[..., ia] = x[..., ia] * cos - x[..., ib] * sin
    y[..., ib] = x[..., ib] * cos + x[..., ia] * sin
    return y


def _check_rounded(got, want, size, terms):
    """got is `want` (64 bits) computed with `terms` fp32 roundings of values up to `size`, rounded once."""
    half = torch.finfo(got.dtype).eps / 2
    tol = half * want.abs() * (1 + terms * 2.0 ** -24) + terms * 2.0 ** -24 * size
    err = (got.double() - want).abs()
    assert torch.isfinite(got.double()).all() and (err <= tol).all(), float((err / tol.clamp(min=1e-300)).max())


ROPE_CASES = [
    # T, hq, hkv, d, rot, norm, interleaved, dtype, first position
    (1, 28, 4, 128, 128, False, False, BF, 0),
    (33, 28, 4, 128, 128, False, False, BF, 131071),
    (7, 64, 8, 128, 128, True, False, BF, 1 << 20),
    (257, 5, 1, 128, 64, True, True, BF, 12345),
    (100, 4, 2, 64, 64, True, False, F32, 999983),
    (3, 8, 8, 64, 32, False, True, F32, 2**31 - 4),
    (65, 16, 2, 128, 96, True, False, F32, 77),
    (2, 3, 3, 64, 16, True, False, BF, 5),
    (5, 4, 2, 128, 128, False, False, F32, -100003),
    (9, 2, 1, 128, 0, True, False, BF, 0),
    (4000, 4, 2, 128, 128, True, False, BF, 3),
]


@pytest.mark.parametrize("T,hq,hkv,d,rot,norm,inter,dtype,first", ROPE_CASES)
@pytest.mark.parametrize("fused", [False, True])
def test_norm_rope_store(T, hq, hkv, d, rot, norm, inter, dtype, first, fused):
    """The norm's sum of d squares, its root, quotient and two products, the rotation's two products and the sine's
    and cosine's own error (an angle within 2^-31 turns, the sums of terms to 2^-23) come to under 32 fp32
    roundings of values up to sqrt(2) times the row's largest."""
    _say(f"norm_rope {T} tokens {hq}/{hkv}/{d} rot {rot} {dtype}")
    g = torch.Generator(device=DEV).manual_seed(T + d)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)
    if fused:
        qkv = r(T, (hq + 2 * hkv) * d + 16).to(dtype)
        q, k, v = (x.view(T, -1, d) for x in qkv[:, :-16].split([hq * d, hkv * d, hkv * d], dim=1))
    else:
        q, k, v = (r(T, h, d).to(dtype) for h in (hq, hkv, hkv))
    page, pages = 16, -(-T * hkv // 16) + 2
    kp, vp = (r(pages, page, d).to(dtype) for _ in range(2))
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:T * hkv].to(torch.int32).view(T, hkv)
    slots[T // 2, 0] = -1
    slots[T // 3, hkv - 1] = pages * page
    pos = (first + torch.arange(T, device=DEV)).clamp(max=2**31 - 1).to(torch.int32)
    inv = (1e6 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / max(rot, 1))).float() if rot else None
    qw, kw = ((1 + 0.3 * r(d)).to(dtype) if norm else None for _ in range(2))
    kp0, vp0, k0, v0, q0 = kp.clone(), vp.clone(), k.clone(), v.clone(), q.clone()
    out = sg.norm_rope_store(q, k, v, pos, slots, kp, vp, inv_freq=inv, q_weight=qw, k_weight=kw, eps=1e-6,
                             interleaved=inter)
    wq = _plain_rope(q0, qw, pos, inv, 1e-6, inter)
    wk = _plain_rope(k0, kw, pos, inv, 1e-6, inter)
    big = lambda w: 2 ** 0.5 * w.abs().amax(-1, keepdim=True).clamp(min=1e-30)
    terms = 32 if (rot or norm) else 0
    _check_rounded(out, wq, big(wq), terms)
    ok = (slots >= 0) & (slots < pages * page)
    at = slots[ok].long()
    _check_rounded(kp.view(-1, d)[at], wk[ok], big(wk)[ok], terms)
    assert torch.equal(vp.view(-1, d)[at], v0[ok])
    rest = torch.ones(pages * page, dtype=torch.bool, device=DEV)
    rest[at] = False
    assert torch.equal(kp.view(-1, d)[rest], kp0.view(-1, d)[rest])
    assert torch.equal(vp.view(-1, d)[rest], vp0.view(-1, d)[rest])
    assert torch.equal(q, q0) and torch.equal(k, k0)


def test_norm_rope_in_place_and_without_queries():
    _say("norm_rope in place")
    T, hq, hkv, d = 50, 6, 2, 128
    g = torch.Generator(device=DEV).manual_seed(0)
    q, k, v = (torch.randn(T, h, d, generator=g, device=DEV).to(BF) for h in (hq, hkv, hkv))
    inv = (1e4 ** (-torch.arange(0, d, 2, device=DEV) / d)).float()
    pos = torch.arange(T, device=DEV, dtype=torch.int32)
    slots = torch.arange(T * hkv, device=DEV, dtype=torch.int32).view(T, hkv)
    pools = [torch.zeros(8, 16, d, device=DEV, dtype=BF) for _ in range(4)]
    out = sg.norm_rope_store(q, k, v, pos, slots, pools[0], pools[1], inv_freq=inv)
    q2 = q.clone()
    same = sg.norm_rope_store(q2, k, v, pos, slots, pools[2], pools[3], inv_freq=inv, q_out=q2)
    assert same is q2 and torch.equal(q2, out)
    assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])
    for p in pools[2:]:
        p.zero_()
    assert sg.norm_rope_store(None, k, v, pos, slots, pools[2], pools[3], inv_freq=inv) is None
    assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])


# ------------------------------------------------------------------ attention
class Case:
    """A paged cache and a step of new tokens. new: tokens per sequence; rows: rows per segment, theirs included."""

    def __init__(self, new, rows, hq, hkv, d, page, dtype, seed=0, pad=0, spread=1.0, garbage=float("nan")):
        g = torch.Generator(device=DEV).manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device=DEV)
        self.new, self.rows_host, self.hq, self.hkv, self.d, self.page = new, rows, hq, hkv, d, page
        self.T = sum(new) + pad
        counts = [-(-x // page) for x in rows]
        n_pages = sum(counts) + 2
        self.perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        width = max(max(counts), 1) + 1
        self.tables = torch.full((len(rows), width), -7, dtype=torch.int32, device=DEV)
        self.k_pages = torch.full((n_pages, page, d), garbage, device=DEV).to(dtype)
        self.v_pages = torch.full((n_pages, page, d), garbage, device=DEV).to(dtype)
        self.k, self.v, at = [], [], 0
        for s, n in enumerate(rows):
            ids = self.perm[at:at + counts[s]]
            at += counts[s]
            self.tables[s, :counts[s]] = ids
            k, v = (r(n, d) * spread).to(dtype), r(n, d).to(dtype)
            slot = (ids.long()[:, None] * page + torch.arange(page, device=DEV)).flatten()[:n]
            self.k_pages.view(-1, d)[slot] = k
            self.v_pages.view(-1, d)[slot] = v
            self.k.append(k)
            self.v.append(v)
        self.q = r(self.T, hq, d).to(dtype)
        self.rows = _i32(rows)
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        self.cu = _i32(cu)

    def call(self, max_new=None, **kw):
        return sg.paged_attention(self.q, self.k_pages, self.v_pages, self.tables, self.rows, self.cu, self.hkv,
                                  max_new=max_new or max(max(self.new), 1), **kw)

    def want(self, causal=True, scale=None):
        """out, lse, sum of p |v| / sum p, largest sum |q_d k_d| per row, rows seen; all in 64 bits."""
        G = self.hq // self.hkv
        scale = scale or 1 / math.sqrt(self.d)
        shape = (self.T, self.hq)
        out = torch.zeros(*shape, self.d, dtype=torch.float64, device=DEV)
        A = torch.zeros_like(out)
        lse = torch.full(shape, -math.inf, dtype=torch.float64, device=DEV)
        big = torch.zeros(shape, dtype=torch.float64, device=DEV)
        seen = torch.zeros(shape, dtype=torch.float64, device=DEV)
        t0 = 0
        for b, n in enumerate(self.new):
            for h in range(self.hkv):
                k, v = self.k[b * self.hkv + h].double(), self.v[b * self.hkv + h].double()
                L = k.shape[0]
                if not (n and L):
                    continue
                mask = None
                if causal:
                    mask = torch.arange(L, device=DEV)[None] > L - n + torch.arange(n, device=DEV)[:, None]
                for i in range(h * G, (h + 1) * G):
                    q = self.q[t0:t0 + n, i].double()
                    y = q @ k.T * scale
                    ab = q.abs() @ k.abs().T
                    if mask is not None:
                        y = y.masked_fill(mask, -math.inf)
                        ab = ab.masked_fill(mask, 0)
                    z = torch.logsumexp(y, 1)
                    p = torch.exp(y - torch.where(z == -math.inf, torch.zeros_like(z), z)[:, None])
                    out[t0:t0 + n, i], A[t0:t0 + n, i] = p @ v, p @ v.abs()
                    lse[t0:t0 + n, i], big[t0:t0 + n, i] = z, ab.amax(1)
                    seen[t0:t0 + n, i] = L
            t0 += n
        return out, lse, A, big, seen, scale

    def check(self, out, lse, causal=True, scale=None, only=None):
        """only: the tokens that are compared (all of them otherwise)."""
        want, wlse, A, big, seen, scale = self.want(causal, scale)
        n = sum(self.new)
        only = torch.ones(n, dtype=torch.bool, device=DEV) if only is None else only[:n]
        blind = wlse[:n] == -math.inf
        fine = torch.where(blind, torch.zeros_like(wlse[:n]), wlse[:n])
        delta = 2.0 ** -21 * abs(scale) * big[:n] + 2.0 ** -22 * (1 + abs(scale) * big[:n])
        prob = 2.0 ** -8 if self.q.dtype == BF and out.dtype == BF else 2.0 ** -24
        half = torch.finfo(out.dtype).eps / 2
        tol = ((2 * delta + prob + (seen[:n] / 4 + 64) * 2.0 ** -24)[..., None] * A[:n]
               + half * want[:n].abs() * (1 + 2.0 ** -8))
        err = (out[:n].double() - want[:n]).abs()
        assert torch.isfinite(out[:n][only].double()).all()
        assert (err <= tol)[only].all(), f"worst {float((err / tol.clamp(min=1e-300)).max())} of the tolerance"
        if lse is not None:
            assert torch.equal((lse[:n] == -math.inf)[only], blind[only])
            got = torch.where(blind, torch.zeros_like(fine), lse[:n].double())
            assert ((got - fine).abs() <= delta + 2.0 ** -21 * (1 + fine.abs()))[only].all()


ATTN_CASES = [
    # new per sequence, rows per segment, hq, hkv, d, page, dtype
    ([1], [1], 1, 1, 128, 16, BF),
    ([1], [17, 300], 14, 2, 128, 16, BF),
    ([1, 1, 1], [5, 64, 1000, 33, 4097, 2], 8, 2, 64, 32, BF),
    ([1, 0, 2, 1], [0, 9, 44, 5, 2, 700, 1, 1], 16, 2, 128, 64, BF),   # an empty segment, a sequence without tokens
    ([2], [40000], 16, 1, 128, 128, BF),                                # a long axis over many workers
    ([4, 1, 3], [129, 130, 128, 127, 7, 513], 14, 2, 128, 16, BF),       # 28 rows
    ([3], [1], 7, 1, 128, 16, BF),                                       # two tokens see nothing
    ([9, 5], [600, 3, 77, 5], 14, 2, 128, 16, BF),                       # blind tokens in a larger tile
    ([100], [100, 1003], 14, 2, 128, 64, BF),
    ([300, 1, 0, 40], [300, 2000, 800, 1, 64, 5000, 40, 41], 10, 2, 128, 128, BF),
    ([1500], [1900, 1500], 32, 2, 128, 256, BF),
    ([200], [9000], 3, 1, 64, 1024, BF),
    ([77, 130], [99, 500], 9, 1, 64, 16, BF),
    ([1], [77, 3000], 2, 2, 64, 16, F32),
    ([1, 2], [700, 1], 9, 1, 128, 32, F32),
    ([50, 3], [1000, 90, 3, 0], 8, 2, 64, 16, F32),
    ([70], [70, 400], 4, 2, 128, 16, F32),
    ([260], [8000], 16, 1, 128, 64, F32),
    ([1] * 40, [(i * 137) % 900 for i in range(80)], 16, 2, 128, 16, BF),
    ([2] * 130, [(i * 31) % 200 for i in range(260)], 2, 2, 64, 16, BF),  # more segments than a workgroup has threads
]


@pytest.mark.parametrize("case", ATTN_CASES)
@pytest.mark.parametrize("causal", [True, False])
def test_paged_attention(case, causal):
    new, rows, hq, hkv, d, page, dtype = case
    _say(f"paged_attention new {new[:6]} rows {rows[:6]} {hq}/{hkv}/{d} page {page} {dtype} causal {causal}")
    c = Case(new, rows, hq, hkv, d, page, dtype, seed=len(rows) + d, pad=3)
    for out_dtype in (BF, F32):
        out = torch.full((c.T, hq, d), 7.0, device=DEV, dtype=out_dtype)
        lse = torch.full((c.T, hq), 7.0, device=DEV)
        c.call(causal=causal, out=out, lse=lse, out_dtype=out_dtype)
        c.check(out, lse, causal)
        n = sum(new)
        assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()  # tokens of nobody


@pytest.mark.parametrize("new,rows,hq,hkv,dtype", [
    ([21], [56783], 5, 1, BF),               # one tile of 105 rows, hundreds of parts
    ([7, 9], [9000, 9003, 40, 12345], 16, 2, F32),
    ([128, 100], [2000] * 8, 28, 4, BF),     # about as many parts as a lane has under way, tiles of fewer rows
    ([6] * 20, [3000] * 40, 16, 2, BF),
])
def test_paged_attention_of_many_parts(new, rows, hq, hkv, dtype):
    _say(f"many parts {new[:3]} over {rows[:3]} {dtype}")
    c = Case(new, rows, hq, hkv, 128, 64, dtype, seed=7)
    out, lse = c.call(out_dtype=F32)
    c.check(out, lse)
    again = c.call(out_dtype=F32)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("dtype,out_dtype,d", [(BF, BF, 128), (BF, F32, 128), (BF, BF, 64), (F32, F32, 64),
                                               (F32, BF, 128)])
def test_paged_attention_of_many_prompts(dtype, out_dtype, d):
    """More tiles than workers: each does several, one after the other, and a value that is not finite in one tile
    stays out of the others."""
    new = [40, 33, 0, 70, 5, 1] * 50
    rows = [n + (17 * i) % 150 for i, n in enumerate(x for n in new for x in (n, n))]
    _say(f"many prompts {dtype} -> {out_dtype} d {d}")
    c = Case(new, rows, 16, 2, d, 32, dtype, seed=d)
    out, lse = c.call(out_dtype=out_dtype)
    c.check(out, lse)
    t0 = 0
    want = out.clone()
    for b, n in enumerate(new):
        for h in range(2):
            seg = 2 * b + h
            if n >= 33 and seg % 3 == 0:
                row, col = rows[seg] - n + n // 2, (7 * seg) % d  # the row of new token n / 2
                page = int(c.tables[seg, row // 32])
                c.v_pages[page, row % 32, col] = float("inf")
                want[t0 + n // 2:t0 + n, 8 * h:8 * h + 8, col] = float("nan")
        t0 += n
    out, lse2 = c.call(out_dtype=out_dtype)
    assert torch.equal(lse, lse2)
    seen = want.isnan()
    assert not torch.isfinite(out[seen]).any() and torch.equal(out[~seen], want[~seen])


@pytest.mark.parametrize("new", [[1], [30]])
@pytest.mark.parametrize("spread", [12.0, 0.0])
def test_paged_attention_far_logits(new, spread):
    """Logits of several hundred (the running reference moves far), and all equal."""
    _say(f"far logits {new} {spread}")
    c = Case(new, [3000, 2999], 14, 2, 128, 64, BF, seed=9, spread=spread)
    c.k_pages.mul_(4.0 if spread else 1.0)
    c.k = [k * 4 if spread else k for k in c.k]
    for od in (BF, F32):
        out, lse = c.call(out_dtype=od)
        c.check(out, lse)


@pytest.mark.parametrize("new", [[1], [3], [40]])
def test_paged_attention_rising_logits(new):
    """Each key's logit is far above all before it: every step moves the reference."""
    _say(f"rising {new}")
    c = Case(new, [900], 8, 1, 128, 16, BF, seed=2)
    for s in range(1):
        k = (torch.arange(900, device=DEV)[:, None] * 0.5 * torch.sign(c.q[0, 0].float())[None]).to(BF)
        slot = (c.perm[:57].long()[:, None] * 16 + torch.arange(16, device=DEV)).flatten()[:900]
        c.k_pages.view(-1, 128)[slot] = k
        c.k[s] = k
    c.q[:] = c.q[0, 0]
    out, lse = c.call(out_dtype=F32)
    c.check(out, lse)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new", [[1, 1], [20, 70]])
def test_paged_attention_scale_and_bounds(dtype, new):
    """A given scale (negative too), max_new above the longest, no lse."""
    _say(f"scale {dtype} {new}")
    c = Case(new, [90, 200, 300, 71], 6, 2, 64, 16, dtype, seed=4)
    for scale in (0.3, -0.11):
        out, none = c.call(max_new=max(new) + 500, scale=scale, with_lse=False)
        assert none is None
        c.check(out, None, scale=scale)


@pytest.mark.parametrize("new", [[1], [60]])
def test_paged_attention_bad_pages_read_as_zeros(new):
    """Table entries that are no page of the pool count as pages of zero rows."""
    _say(f"bad pages {new}")
    c = Case(new, [500, 300], 8, 2, 128, 16, BF, seed=6)
    for s, j, bad in ((0, 3, -1), (0, 20, c.k_pages.shape[0]), (1, 0, 2**31 - 1), (1, 5, -2**31)):
        c.tables[s, j] = bad
        c.k[s][16 * j:16 * j + 16] = 0
        c.v[s][16 * j:16 * j + 16] = 0
    out, lse = c.call(out_dtype=F32)
    c.check(out, lse)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,new", [(2, [5, 1]), (6, [6, 3]), (8, [40, 33])])
def test_paged_attention_values_of_tokens_to_come(hq, new, dtype, bad):
    """Keys and values that are not finite reach no token that does not see their row (16, 48 and 128 rows a tile);
    the tokens that see them come out not finite."""
    _say(f"not finite {bad} {dtype} {new}")
    c = Case(new, [70, 200, 33, 1000], hq, 2, 128, 16, dtype, seed=13)
    n = new[0]
    at = n - 2  # the token before the last of the first sequence
    for s in (0, 1):
        row = c.rows_host[s] - n + at
        page = int(c.tables[s, row // 16])
        c.v_pages[page, row % 16, 5:9] = bad
        c.k_pages[page, row % 16, 3] = float("nan")
    for od in (BF, F32):
        out, lse = c.call(out_dtype=od)
        rest = torch.ones(c.T, dtype=torch.bool, device=DEV)
        rest[at:n] = False
        c.check(out, lse, only=rest)
        assert not torch.isfinite(lse[at:n]).any() and not torch.isfinite(out[at:n]).any()


def test_paged_attention_cuts_lengths_to_the_buffers():
    """rows beyond the table, cu_new beyond T, a chunk beyond max_new: cut, and the rest left alone."""
    _say("cut lengths")
    c = Case([5], [64, 64], 4, 2, 64, 16, BF, seed=8)
    c.tables = c.tables[:, :4].contiguous()
    c.rows.fill_(2**31 - 1)
    c.cu.copy_(_i32([-4, 5]))
    out, lse = c.call()
    c.check(out, lse)
    c.cu.copy_(_i32([0, 2**30]))
    out2, _ = c.call()
    assert torch.equal(out, out2)
    kept = torch.full_like(out, 3.0)
    c.call(max_new=2, out=kept)
    assert torch.equal(kept[:2], out[:2]) or (kept[:2].float() - out[:2].float()).abs().max() < 0.05
    assert (kept[2:] == 3.0).all()


@pytest.mark.parametrize("new,rows,hq,hkv", [([1, 1], [30000, 100, 7, 9000], 14, 2),
                                             ([200, 9], [5000, 700, 40, 9], 14, 2)])
def test_paged_attention_repeats_bit_for_bit(new, rows, hq, hkv):
    _say(f"repeat {new}")
    c = Case(new, rows, hq, hkv, 128, 64, BF, seed=3)
    a = c.call(out_dtype=F32)
    b = c.call(out_dtype=F32)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_paged_attention_of_nothing():
    c = Case([0, 0], [5, 0], 2, 1, 64, 16, BF)
    out, lse = c.call(max_new=4)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)


# ------------------------------------------------------------------ together
def _serve_state(B, hkv, page, max_pages, n_pages, d, dtype):
    return dict(rows=torch.zeros(B * hkv, dtype=torch.int32, device=DEV), head=_i32([0]),
                tables=torch.full((B * hkv, max_pages), -1, dtype=torch.int32, device=DEV),
                free=torch.randperm(n_pages, device=DEV).to(torch.int32),
                k=torch.full((n_pages, page, d), float("nan"), device=DEV, dtype=dtype),
                v=torch.full((n_pages, page, d), float("nan"), device=DEV, dtype=dtype))


def test_compressed_cache_in_pages_decodes_as_the_ragged_one():
    """compress_layer, its rows into pages, then one new token: the paged attention against decode_attention
    over the ragged cache with the token's rows appended; and the token's rows given up again."""
    _say("compress -> pages -> attention")
    B, hq, hkv, d, C, w, page = 2, 14, 2, 128, 2000, 32, 32
    g = torch.Generator(device=DEV).manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV).to(BF)
    budgets = [700, 300]
    res = sg.compress_layer(r(B, hq, w, d), r(B, hkv, C, d), r(B, hkv, C, d), budgets, pool_kernel=7, b_sink=4,
                            b_window=64)
    st = _serve_state(B, hkv, page, 64, 200, d, BF)
    up = sg.page_update(st["rows"], _i32(budgets * B), st["tables"], st["free"], st["head"], page_size=page,
                        n_slots=sum(budgets) * B, by_segment=True, rows_out=st["rows"], head_out=st["head"])
    assert torch.equal(up["cu"].long(), res["offsets"])
    sg.paged_store(res["k_c"], res["v_c"], up["slots"], st["k"], st["v"])
    step = sg.page_update(st["rows"], _i32([1, 1]), st["tables"], st["free"], st["head"], page_size=page, n_slots=B)
    q, k, v = r(B, hq, d), r(B, hkv, d), r(B, hkv, d)
    inv = (1e6 ** (-torch.arange(0, d, 2, device=DEV) / d)).float()
    pos = _i32([C, C])
    qr = sg.norm_rope_store(q, k, v, pos, step["slots"], st["k"], st["v"], inv_freq=inv)
    out, lse = sg.paged_attention(qr, st["k"], st["v"], st["tables"], step["rows"], step["cu"], hkv, max_new=1,
                                  out_dtype=F32)
    k_new, v_new = torch.zeros(B, hkv, 8, d, device=DEV, dtype=BF), torch.zeros(B, hkv, 8, d, device=DEV, dtype=BF)
    rows_k = st["k"].view(-1, d)[step["slots"].long()]
    sg.append_kv(qr, rows_k.contiguous(), v, k_new, v_new, 0)
    ref, ref_lse = sg.decode_attention(qr, res["k_c"], res["v_c"], res["offsets"], res["offsets_host"], hkv,
                                       out_dtype=F32, k_new=k_new, v_new=v_new, n_new=1)
    # each is within (2 delta + (701 / 4 + 64) 2^-24) A, delta about 5e-6 and A about 1 here: 3e-5, both 6e-5
    assert (out - ref).abs().max() < 6e-5 and (lse - ref_lse).abs().max() < 2e-5
    back = sg.page_update(step["rows"], _i32([-1, -1]), st["tables"], st["free"], step["head"], page_size=page,
                          n_slots=0)
    assert torch.equal(back["rows"], st["rows"]) and torch.equal(back["head"], st["head"])
    assert int(back["status"]) == 0


@pytest.mark.parametrize("chunks", [[5, 1, 1], [70, 3, 40]])
def test_steps_against_the_whole_sequence(chunks):
    """A sequence fed in chunks gives the outputs of one pass over all its tokens."""
    _say(f"steps {chunks}")
    B, hq, hkv, d, page = 3, 8, 2, 64, 16
    g = torch.Generator(device=DEV).manual_seed(7)
    n = sum(chunks)
    q, k, v = (torch.randn(B, n, h, d, generator=g, device=DEV) for h in (hq, hkv, hkv))
    inv = (1e4 ** (-torch.arange(0, d, 2, device=DEV) / d)).float()
    wts = [1 + 0.1 * torch.randn(d, generator=g, device=DEV) for _ in range(2)]
    outs = []
    for plan in (chunks, [n]):
        st = _serve_state(B, hkv, page, 16, 100, d, F32)
        got, done = [], 0
        for m in plan:
            up = sg.page_update(st["rows"], _i32([m] * B), st["tables"], st["free"], st["head"], page_size=page,
                                n_slots=B * m, rows_out=st["rows"], head_out=st["head"])
            cut = lambda x: x[:, done:done + m].reshape(B * m, -1, d)
            pos = (done + torch.arange(m, device=DEV, dtype=torch.int32)).repeat(B)
            qr = sg.norm_rope_store(cut(q), cut(k), cut(v), pos, up["slots"], st["k"], st["v"], inv_freq=inv,
                                    q_weight=wts[0], k_weight=wts[1])
            out, _ = sg.paged_attention(qr, st["k"], st["v"], st["tables"], up["rows"], up["cu"], hkv, max_new=m)
            got.append(out.view(B, m, hq, d))
            done += m
        outs.append(torch.cat(got, 1))
    assert (outs[0] - outs[1]).abs().max() < 1e-5


def test_captured_steps_replay_with_new_lengths():
    """One captured step (pages, norm and rotation, attention) replayed while the cache grows, against eager
    steps on a second cache, with eager work between the replays; then two captures with workspaces of their own."""
    _say("captured steps")
    B, hq, hkv, d, page, T = 4, 14, 2, 128, 16, 8
    g = torch.Generator(device=DEV).manual_seed(5)
    inv = (1e6 ** (-torch.arange(0, d, 2, device=DEV) / d)).float()
    a, b = (_serve_state(B, hkv, page, 64, 600, d, BF) for _ in range(2))
    b["free"].copy_(a["free"])
    io = dict(q=torch.zeros(T, hq, d, device=DEV, dtype=BF), k=torch.zeros(T, hkv, d, device=DEV, dtype=BF),
              v=torch.zeros(T, hkv, d, device=DEV, dtype=BF), pos=_i32([0] * T), add=_i32([0] * B))
    ws = sg.alloc_workspace(sg.paged_attention_workspace_size(io["q"], hkv, B, max_new=T), DEV)

    def step(st, ws):
        up = sg.page_update(st["rows"], io["add"], st["tables"], st["free"], st["head"], page_size=page, n_slots=T,
                            rows_out=st["rows"], head_out=st["head"])
        qr = sg.norm_rope_store(io["q"], io["k"], io["v"], io["pos"], up["slots"], st["k"], st["v"], inv_freq=inv)
        out = torch.zeros(T, hq, d, device=DEV, dtype=BF)
        lse = torch.zeros(T, hq, device=DEV)
        return sg.paged_attention(qr, st["k"], st["v"], st["tables"], up["rows"], up["cu"], hkv, max_new=T, out=out,
                                  lse=lse, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a, ws)  # add is 0: nothing changes
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step(a, ws)
    for i, add in enumerate([[2, 1, 3, 2], [8, 0, 0, 0], [1, 1, 1, 1], [-5, 3, 0, 5], [0, 8, 0, 0], [1, 0, 7, 0]]):
        io["add"].copy_(_i32(add))
        for x in ("q", "k", "v"):
            io[x].copy_(torch.randn(io[x].shape, generator=g, device=DEV))
        io["pos"].copy_(torch.randint(0, 5000, (T,), generator=g, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        want, want_lse = step(b, None)
        assert torch.equal(out, want) and torch.equal(lse, want_lse), i
        assert torch.equal(a["rows"], b["rows"]) and torch.equal(a["tables"], b["tables"])
        assert torch.equal(a["k"].view(torch.int16), b["k"].view(torch.int16))


def test_another_stream():
    """Calls given a stream wait for nothing else and leave their results on it."""
    _say("another stream")
    c = Case([40, 1], [500, 40, 300, 77], 14, 2, 128, 16, BF, seed=12)
    want, want_lse = c.call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, lse = c.call(stream=side)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    out, _ = c.call(stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(out, want)


def test_page_update_of_the_most_segments():
    """4096 segments by segment: lengths and prefix sums fill the most LDS a call takes."""
    _say("page_update 4096 segments")
    rows = [(i * 13) % 40 for i in range(4096)]
    add = [(i * 29) % 50 - 12 for i in range(4096)]
    tables, free, head = _start(rows, 16, 6, 20000, 2)
    _update_both(rows, add, tables, free, head, 16, sum(max(x, 0) for x in add) + 3, 1, True)


def test_pools_beyond_4_gib():
    """Pages whose bytes and rows lie past 2^32 bytes of the pool: stores, rotation and both attention kernels."""
    _say("pools beyond 4 GiB")
    d, page, hq, hkv = 128, 256, 8, 2
    n_pages = (5 << 30) // (page * d * 2)
    kp, vp = (torch.empty(n_pages, page, d, dtype=BF, device=DEV) for _ in range(2))
    for new in ([1, 2], [40, 9]):
        c = Case(new, [300, 700, 257, 512], hq, hkv, d, page, BF, seed=21)
        far = c.tables.clone()
        used = c.tables >= 0
        far[used] = n_pages - 1 - c.tables[used]
        slot = lambda s: (far[s].long()[:, None] * page + torch.arange(page, device=DEV)).flatten()[:c.rows_host[s]]
        for s in range(4):
            sg.paged_store(c.k[s], c.v[s], slot(s).to(torch.int32), kp, vp)
            assert torch.equal(kp.view(-1, d)[slot(s)], c.k[s])
        c.k_pages, c.v_pages, c.tables = kp, vp, far
        out, lse = c.call(out_dtype=F32)
        c.check(out, lse)
    k = torch.randn(3, hkv, d, device=DEV).to(BF)
    slots = (n_pages * page - 1 - torch.arange(6, device=DEV)).to(torch.int32).view(3, hkv)
    sg.norm_rope_store(None, k, k, _i32([0, 0, 0]), slots, kp, vp)
    assert torch.equal(kp.view(-1, d)[slots.flatten().long()], k.view(-1, d))


def test_two_calls_at_once():
    """Calls on two streams with a workspace each, overlapping, against the same calls one after the other."""
    _say("two at once")
    cases = [Case([1, 1], [30000, 20000, 3000, 50], 14, 2, 128, 64, BF, seed=31),
             Case([300, 77], [3000, 5000, 300, 77], 14, 2, 128, 16, BF, seed=32)]
    want = [c.call() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    ws = [sg.alloc_workspace(sg.paged_attention_workspace_size(c.q, c.hkv, 2, max_new=max(c.new)), DEV) for c in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        got = [c.call(workspace=w, stream=s) for c, w, s in zip(cases, ws, streams)]
        torch.cuda.synchronize()
        for (o, l), (wo, wl) in zip(got, want):
            assert torch.equal(o, wo) and torch.equal(l, wl)


def test_two_captured_calls_share_a_workspace():
    """Two captured graphs with one workspace, replayed in turn on one stream, with eager calls between."""
    _say("two graphs, one workspace")
    cases = [Case([1, 1], [9000, 20000, 3000, 50], 14, 2, 128, 64, BF, seed=41),
             Case([130, 7], [3000, 500, 300, 77], 14, 2, 128, 16, BF, seed=42)]
    want = [c.call() for c in cases]
    ws = sg.alloc_workspace(max(sg.paged_attention_workspace_size(c.q, c.hkv, 2, max_new=max(c.new)) for c in cases),
                            DEV)
    graphs, outs = [], []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        out, lse = torch.zeros_like(c.q), torch.zeros(c.T, c.hq, device=DEV)
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            c.call(workspace=ws, out=out, lse=lse)
        graphs.append(g)
        outs.append((out, lse))
    for _ in range(4):
        for g, c, (out, lse), (wo, wl) in zip(graphs, cases, outs, want):
            out.zero_()
            g.replay()
            eager = c.call()
            torch.cuda.synchronize()
            assert torch.equal(out, wo) and torch.equal(lse, wl) and torch.equal(eager[0], wo)


def test_shared_pages():
    """Two sequences whose tables name the same pages (a common prompt) read the same rows."""
    _say("shared pages")
    c = Case([1, 3], [500, 90, 500, 90], 8, 2, 128, 16, BF, seed=51)
    c.tables[2:] = c.tables[:2]
    c.k[2:], c.v[2:] = c.k[:2], c.v[:2]
    out, lse = c.call(out_dtype=F32)
    c.check(out, lse)


@pytest.mark.parametrize("hq,new", [(2, [3]), (4, [40])])
def test_many_segments(hq, new):
    """600 sequences: more tiles than workers, most of a token, one of many."""
    _say(f"many segments {new}")
    n = [1 if i % 7 else 0 for i in range(600)]
    n[300] = new[0]
    c = Case(n, [(i * 53) % 70 + n[i // 2] for i in range(1200)], hq, 2, 64, 16, BF, seed=61)
    out, lse = c.call(out_dtype=F32)
    c.check(out, lse)


def test_a_step_without_pages_does_nothing():
    """Too few pages: the step's calls that follow store nothing, attend to nothing and change no length."""
    _say("no pages")
    B, hq, hkv, d, page = 2, 4, 2, 64, 16
    st = _serve_state(B, hkv, page, 8, 3, d, F32)
    up = sg.page_update(st["rows"], _i32([1, 1]), st["tables"], st["free"], st["head"], page_size=page, n_slots=B,
                        rows_out=st["rows"], head_out=st["head"])
    assert int(up["status"]) == sg.PAGES_SHORT and (up["slots"] == -1).all() and not up["cu"].any()
    x = torch.randn(B, hkv, d, device=DEV)
    q = sg.norm_rope_store(torch.randn(B, hq, d, device=DEV), x, x, _i32([0, 0]), up["slots"], st["k"], st["v"])
    assert st["k"].isnan().all() and st["v"].isnan().all()
    out = torch.full_like(q, 5.0)
    sg.paged_attention(q, st["k"], st["v"], st["tables"], st["rows"], up["cu"], hkv, max_new=1, out=out)
    assert (out == 5.0).all() and not st["rows"].any() and int(st["head"]) == 0


@pytest.mark.parametrize("new", [[1], [20]])
def test_table_of_repeated_pages_past_2_to_25_rows(new):
    """A segment of 40 million rows whose table names the same 64 pages over and over: its softmax is that of the
    pages' rows, each many times, so out is that of one round of them and lse larger by the log of the rounds.
    Equal parts of the sums round together: the tolerances are those of one round with this many rows."""
    _say(f"long table {new}")
    d, page, P, rounds = 64, 1024, 64, 620
    g = torch.Generator(device=DEV).manual_seed(0)
    kp, vp = (torch.randn(P, page, d, generator=g, device=DEV).to(BF) for _ in range(2))
    tables = torch.arange(P, dtype=torch.int32, device=DEV).repeat(rounds)[None].contiguous()
    q = torch.randn(sum(new), 4, d, generator=g, device=DEV).to(BF)
    rows = _i32([P * page * rounds])
    out, lse = sg.paged_attention(q, kp, vp, tables, rows, _i32([0, len(q)]), 1, max_new=max(new), causal=False,
                                  out_dtype=F32)
    y = q.double().flatten(0, 1) @ kp.view(-1, d).double().T / 8
    want = torch.softmax(y, 1) @ vp.view(-1, d).double()
    wlse = torch.logsumexp(y, 1) + math.log(rounds)
    # a worker adds 79000 rows, 4 at a time per lane group and 16 per product: 2500 roundings at most meet in a sum
    assert (out.double().flatten(0, 1) - want).abs().max() < 2500 * 2.0 ** -24 * 1.0 + 2e-5
    assert (lse.double().flatten() - wlse).abs().max() < 2500 * 2.0 ** -24 + 2e-5


@pytest.mark.parametrize("new,rows,hq,hkv,d", [
    ([1, 1], [700, 30000, 1, 64], 16, 2, 128),          # 8 rows of 16
    ([1, 2, 1], [90, 4000, 333], 16, 1, 64),            # 32 rows
    ([6, 1, 3], [5000, 129, 7, 700, 16, 90], 16, 2, 128),  # 48 rows
])
def test_paged_attention_of_few_rows_keeps_the_probabilities_bits(new, rows, hq, hkv, d):
    """bf16 output of up to 48 query rows per KV head is the fp32 output rounded once: bit for bit, and within the
    fp32 output's tolerance and half a bf16 step of the 64-bit value."""
    _say(f"probabilities {new} {hq}/{hkv}/{d}")
    c = Case(new, rows, hq, hkv, d, 16, BF, seed=17)
    out, lse = c.call(out_dtype=BF)
    fine, lse2 = c.call(out_dtype=F32)
    c.check(fine, lse2)
    assert torch.equal(out, fine.to(BF)) and torch.equal(lse, lse2)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype,d,rot", [(BF, 128, 64), (F32, 128, 96), (F32, 64, 16), (BF, 64, 32)])
def test_norm_rope_columns_that_do_not_turn(dtype, d, rot, inter):
    """Without a norm the columns from rot on are copied, whatever they hold: infinities, NaN and both zeros bit for
    bit; and the others come out as if those held ordinary values."""
    _say(f"columns that do not turn {dtype} {d}/{rot}")
    g = torch.Generator(device=DEV).manual_seed(rot)
    T, hq, hkv = 9, 5, 2
    q, k, v = (torch.randn(T, h, d, generator=g, device=DEV).to(dtype) for h in (hq, hkv, hkv))
    inv = (1e4 ** (-torch.arange(0, rot, 2, device=DEV) / rot)).float()
    pos = 11 + 1000 * torch.arange(T, device=DEV, dtype=torch.int32)
    slots = torch.arange(T * hkv, device=DEV, dtype=torch.int32).view(T, hkv)
    outs = []
    for odd in (False, True):
        kp, vp = (torch.zeros(2, 16, d, device=DEV, dtype=dtype) for _ in range(2))
        if odd:
            special = torch.tensor([math.inf, -math.inf, math.nan, -0.0, 0.0, 1.0, -2.0], device=DEV).to(dtype)
            for x in (q, k):
                x[..., rot:] = special[torch.randint(0, 7, x[..., rot:].shape, generator=g, device=DEV)]
        out = sg.norm_rope_store(q, k, v, pos, slots, kp, vp, inv_freq=inv, interleaved=inter)
        stored = kp.view(-1, d)[:T * hkv].view(T, hkv, d)
        bits = torch.int16 if dtype == BF else torch.int32
        for got, had in ((out, q), (stored, k)):
            assert torch.equal(got[..., rot:].contiguous().view(bits), had[..., rot:].contiguous().view(bits))
        outs.append((out[..., :rot], stored[..., :rot]))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("first", [0, 131072, 2**31 - 3000, -3000])
def test_norm_rope_angles(first, inter):
    """Pairs (1, 0) turn into (cos t, sin t) with no rounding of their own, so what comes out is the cosine and sine:
    off by an angle of 2^-31 turns at most (their slope is 1 at most) and by their rounding to fp32, half a step of the
    value. The reference takes the exact product of position and frequency in 80 bits and its sine in 64."""
    _say(f"angles from {first}")
    np = pytest.importorskip("numpy")
    T, d = 3000, 128
    half = d // 2
    pos = first + torch.arange(T, dtype=torch.int64)
    inv = (1e6 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float()
    k = torch.zeros(T, 1, d, device=DEV)
    k[..., 0::2] = 1.0 if inter else 0.0
    if not inter:
        k[..., :half] = 1.0
    kp, vp = (torch.zeros(-(-T // 16), 16, d, device=DEV) for _ in range(2))
    slots = torch.arange(T, device=DEV, dtype=torch.int32)[:, None].contiguous()
    sg.norm_rope_store(None, k, k, pos.to(torch.int32).to(DEV), slots, kp, vp, inv_freq=inv.to(DEV), interleaved=inter)
    out = kp.view(-1, d)[:T].cpu().double()
    cos, sin = (out[:, 0::2], out[:, 1::2]) if inter else (out[:, :half], out[:, half:])
    # a 31-bit position by a 24-bit frequency is exact in 80 bits; so is nearly its rest of whole turns (2^-64 2^31)
    pi2 = np.longdouble(2 * math.pi) + np.longdouble(2.449293598294706e-16)
    t = pos.numpy().astype(np.longdouble)[:, None] * inv.numpy().astype(np.longdouble)[None]
    t = torch.from_numpy((t - np.rint(t / pi2) * pi2).astype(np.float64))
    for got, want in ((cos, torch.cos(t)), (sin, torch.sin(t))):
        tol = 2.0 ** -24 * want.abs() + 2 * math.pi * 2.0 ** -31
        err = (got - want).abs()
        assert (err <= tol).all(), float((err / tol).max())


def test_norm_rope_of_more_tokens_than_a_launch_holds():
    """2^26 + 37 tokens, a wave each, are more threads than one launch takes; tokens around each power of two from 2^24
    on are compared, and the slots of the others are -1."""
    _say("norm_rope of 2^26 + 37 tokens")
    T, d = 2**26 + 37, 64
    g = torch.Generator(device=DEV).manual_seed(4)
    k = torch.zeros(T, 1, d, device=DEV, dtype=BF)
    pos = torch.zeros(T, device=DEV, dtype=torch.int32)
    slots = torch.full((T, 1), -1, device=DEV, dtype=torch.int32)
    some = torch.tensor([0, *(2**i + j for i in (24, 25, 26) for j in (-1, 0, 1)), T - 1], device=DEV)
    k[some] = torch.randn(len(some), 1, d, generator=g, device=DEV).to(BF)
    pos[some] = (some % 100003).to(torch.int32)
    slots[some, 0] = torch.arange(len(some), device=DEV, dtype=torch.int32)
    inv = (1e4 ** (-torch.arange(0, d, 2, device=DEV) / d)).float()
    kp, vp = (torch.zeros(1, 16, d, device=DEV, dtype=BF) for _ in range(2))
    out = sg.norm_rope_store(k, k, k, pos, slots, kp, vp, inv_freq=inv)
    small = torch.zeros_like(kp)
    want = sg.norm_rope_store(k[some], k[some], k[some], pos[some], slots[some], small, vp.clone(), inv_freq=inv)
    assert torch.equal(out[some], want) and torch.equal(kp, small)
    assert torch.equal(vp[0, :len(some)], k[some, 0])
    _check_rounded(want, _plain_rope(k[some], None, pos[some], inv, 0.0, False),
                   2 ** 0.5 * k[some].double().abs().amax(-1, keepdim=True), 32)


def test_the_default_streams_handle():
    """stream=0 is the default stream: the call comes after what was sent there before, and before what comes next."""
    _say("stream 0")
    c = Case([40, 1], [500, 40, 300, 77], 14, 2, 128, 16, BF, seed=12)
    want, want_lse = c.call()
    q = c.q.clone()
    ws = sg.alloc_workspace(sg.paged_attention_workspace_size(q, 2, 2, max_new=40), DEV)
    out, lse = torch.zeros_like(want), torch.zeros_like(want_lse)
    for _ in range(3):
        c.q.zero_()
        out.zero_()
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)  # about 10 ms, far longer than the call
        c.q.copy_(q)
        c.call(stream=0, out=out, lse=lse, workspace=ws)
        got = out.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(lse, want_lse)


def test_tensors_are_marked_on_torchs_streams_alone(monkeypatch):
    """A mark outlives the call: torch uses its stream when the tensor is freed. So the tensors of a call are marked on
    a torch.cuda.Stream, and not on a raw handle, whose stream may be gone by then."""
    _say("marks")
    c = Case([3], [40], 4, 1, 64, 16, BF)
    side = torch.cuda.Stream()
    ws = sg.alloc_workspace(sg.paged_attention_workspace_size(c.q, 1, 1, max_new=3), DEV)
    side.wait_stream(torch.cuda.current_stream())
    marked, mark = [], torch.Tensor.record_stream
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: (marked.append(t.data_ptr()), mark(t, s)) and None)
    c.call(stream=side.cuda_stream, workspace=ws)
    assert not marked
    c.call(stream=side, workspace=ws)
    assert {t.data_ptr() for t in (c.q, c.k_pages, c.v_pages, c.tables, c.rows, c.cu, ws)} == set(marked)
    side.synchronize()


def test_page_update_refuses_results_over_other_arguments():
    """rows_out over add, or over a part of rows, would be written by one workgroup while another still reads it."""
    _say("overlapping results")
    pool = _i32([0] * 64)
    rows, add, head = pool[:8], pool[16:24], pool[32:33]
    tables, free = _i32([[0] * 4] * 8), _i32([1, 2, 3])
    kw = dict(page_size=16, n_slots=4, by_segment=True)
    cu, slots = _i32([0] * 9), _i32([0] * 4)
    for bad in (dict(rows_out=add), dict(rows_out=pool[4:12]), dict(head_out=rows[:1]), dict(head_out=free[2:3]),
                dict(rows_out=pool[40:48], head_out=pool[44:45]), dict(rows_out=cu[:8], cu=cu),
                dict(head_out=slots[:1], slots=slots), dict(rows_out=tables.view(-1)[8:16])):
        with pytest.raises(sg.SgdkvError) as e:
            sg.page_update(rows, add, tables, free, head, **kw, **bad)
        assert e.value.status == sg.ERR_INVALID_ARG and "overlaps" in e.value.message
    for good in (dict(rows_out=rows, head_out=head), dict(rows_out=pool[40:48], head_out=pool[48:49])):
        up = sg.page_update(rows, add, tables, free, head, **kw, **good)
        assert int(up["status"]) == 0 and not up["rows"].any()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("hq,new,rows,dtype", [
    (2, [5, 1], [70, 200, 33, 1000], BF),        # 5 query rows of 16
    (6, [6, 3], [9000, 61, 33, 1000], BF),       # 18 of 32, a segment cut into many parts
    (6, [16, 1], [130, 12000, 33, 40], BF),      # 48
    (8, [40, 33], [70, 9000, 33, 1000], BF),     # 128
    (2, [13, 1], [9000, 200, 33, 90], F32),      # 13 of 16
    (4, [15, 15], [70, 7000, 15, 16], F32),      # 30 of 32
    (8, [40, 33], [7000, 200, 40, 1000], F32),   # 128
])
@pytest.mark.parametrize("d", [64, 128])
def test_paged_attention_values_alone_that_are_not_finite(hq, new, rows, dtype, d, bad):
    """Values that are not finite, keys all finite: not finite are the outputs of exactly their columns of the tokens
    that see their rows; every other output, and every lse, is that of the clean run bit for bit. The rows are those of
    the last two tokens, so that some of a tile's rows see them and others do not; the columns are an odd and an even
    one (both halves of a word), the first and the last."""
    _say(f"values {bad} {dtype} {new} over {rows} d {d}")
    c = Case(new, rows, hq, 2, d, 16, dtype, seed=13)
    n, G = new[0], hq // 2
    for od in (BF, F32):
        clean, clean_lse = c.call(out_dtype=od)
        odd = torch.zeros(clean.shape, dtype=torch.bool, device=DEV)
        saved = c.v_pages.clone()
        for s, token, cols in ((0, n - 2, (5, 8)), (0, n - 1, (0, d - 1)), (1, n - 1, (6, 7)), (1, n - 2, (d - 2,))):
            row = rows[s] - n + token
            page = int(c.tables[s, row // 16])
            for col in cols:
                c.v_pages[page, row % 16, col] = bad
                odd[token:n, s * G:(s + 1) * G, col] = True
        out, lse = c.call(out_dtype=od)
        assert torch.equal(lse, clean_lse)
        assert not torch.isfinite(out[odd]).any() and torch.equal(out[~odd], clean[~odd])
        c.v_pages = saved


@pytest.mark.parametrize("hq,new,max_new,dtype", [(4, 5, 2, BF), (6, 16, 3, BF), (8, 100, 37, BF), (8, 100, 5, BF),
                                                  (4, 16, 7, F32), (4, 90, 33, F32)])
def test_paged_attention_of_the_first_max_new_tokens(hq, new, max_new, dtype):
    """A chunk longer than max_new: its first max_new tokens come out as they do with the rest, within the tolerance
    of the 64-bit values, whichever kernel; the others' out and lse are left alone."""
    _say(f"max_new {max_new} of {new}")
    c = Case([new], [64 + new, 700], hq, 2, 64, 16, dtype, seed=8)
    for od in (BF, F32):
        out = torch.full((c.T, hq, 64), 3.0, device=DEV, dtype=od)
        lse = torch.full((c.T, hq), 3.0, device=DEV)
        c.call(max_new=max_new, out=out, lse=lse, out_dtype=od)
        assert (out[max_new:] == 3.0).all() and (lse[max_new:] == 3.0).all()
        c.check(out, lse, only=torch.arange(c.T, device=DEV) < max_new)


def _in_place_steps(rows, steps, hkv, page, by_segment, width):
    """Calls in a row with rows_out = rows and head_out = head, each against lists of integers."""
    n_pages = sum(-(-r // page) for r in rows) + 3 + sum(sum(-(-max(a, 0) // page) + 1 for a in add) * (
        1 if by_segment else hkv) for add in steps)
    tables, free, head = _start(rows, page, width, n_pages, 11)
    d = dict(rows=_i32(rows), tables=_i32(tables), free=_i32(free), head=_i32([head]))
    state = (rows, tables, free, head)
    for add in steps:
        n_slots = sum(max(a, 0) for a in add) + 2
        want = _plain_update(*state[:1], add, *state[1:], page, n_slots, hkv, by_segment)
        assert want["status"] == 0
        got = sg.page_update(d["rows"], _i32(add), d["tables"], d["free"], d["head"], page_size=page, n_slots=n_slots,
                             by_segment=by_segment, rows_out=d["rows"], head_out=d["head"])
        assert got["rows"] is d["rows"] and got["head"] is d["head"]
        _check_update(got, want)
        state = (want["rows"], want["tables"], want["free_pages"], want["head"])


def test_page_update_by_segment_in_place():
    """The rows of a batch of compressed prompts in place, over many workgroups; then some given back, some taken."""
    _say("page_update by segment in place")
    S = 64
    first = [(i * 977) % 5000 + 17 for i in range(S)]
    second = [-((i * 331) % 900) if i % 3 else (i * 977) % 3000 for i in range(S)]
    _in_place_steps([0] * S, [first, second, [-10000] * S], 1, 16, True, 600)


def test_page_update_of_a_token_each_in_place_with_wide_tables():
    """One token for 512 segments whose tables have 1200 columns: the tables alone make it many workgroups."""
    _say("page_update 512 x 1200 in place")
    rows = [(i * 53) % 3000 for i in range(512)]
    _in_place_steps(rows, [[1] * 64, [1 if i % 5 else -40 for i in range(64)]], 8, 16, False, 1200)


@pytest.mark.parametrize("chunks", [[5, 1, 1], [70, 3, 40]])
def test_steps_against_64_bits(chunks):
    """Steps of page_update, norm_rope_store and paged_attention, each against 64 bits: the stored keys against the
    whole sequence's norm and rotation, the outputs against the softmax over the rows stored so far."""
    _say(f"steps {chunks} in 64 bits")
    B, hq, hkv, d, page = 3, 8, 2, 64, 16
    g = torch.Generator(device=DEV).manual_seed(7)
    n = sum(chunks)
    q, k, v = (torch.randn(B, n, h, d, generator=g, device=DEV) for h in (hq, hkv, hkv))
    inv = (1e4 ** (-torch.arange(0, d, 2, device=DEV) / d)).float()
    wts = [1 + 0.1 * torch.randn(d, generator=g, device=DEV) for _ in range(2)]
    pos = torch.arange(n, device=DEV, dtype=torch.int32)
    wq, wk = (torch.stack([_plain_rope(x[b], w, pos, inv, 1e-6, False) for b in range(B)])
              for x, w in zip((q, k), wts))
    big = lambda w: 2 ** 0.5 * w.abs().amax(-1, keepdim=True)
    st = _serve_state(B, hkv, page, 16, 100, d, F32)
    done = 0
    for m in chunks:
        up = sg.page_update(st["rows"], _i32([m] * B), st["tables"], st["free"], st["head"], page_size=page,
                            n_slots=B * m, rows_out=st["rows"], head_out=st["head"])
        cut = lambda x: x[:, done:done + m].reshape(B * m, -1, d)
        qr = sg.norm_rope_store(cut(q), cut(k), cut(v), pos[done:done + m].repeat(B), up["slots"], st["k"], st["v"],
                                inv_freq=inv, q_weight=wts[0], k_weight=wts[1])
        out, lse = sg.paged_attention(qr, st["k"], st["v"], st["tables"], up["rows"], up["cu"], hkv, max_new=m)
        done += m
        _check_rounded(qr.view(B, m, hq, d), wq[:, done - m:done], big(wq[:, done - m:done]), 32)
        # the attention's reference takes the rotated queries and the rows as they were stored
        c = Case.__new__(Case)
        c.new, c.rows_host, c.hq, c.hkv, c.d, c.T = [m] * B, [done] * (B * hkv), hq, hkv, d, B * m
        c.q, c.k, c.v = qr, [], []
        for s in range(B * hkv):
            at = torch.arange(done, device=DEV)
            slot = st["tables"][s].long()[at // page] * page + at % page
            c.k.append(st["k"].view(-1, d)[slot])
            c.v.append(st["v"].view(-1, d)[slot])
            b, h = divmod(s, hkv)
            _check_rounded(c.k[-1], wk[b, :done, h], big(wk[b, :done, h]), 32)
            assert torch.equal(c.v[-1], v[b, :done, h])
        c.check(out, lse)
