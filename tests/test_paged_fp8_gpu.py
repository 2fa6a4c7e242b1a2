"""The paged per-head cache in 8 bits on an MI355X: rows into pages, norm and rotation, attention of new tokens, each
against a plain implementation in 64 bits, alone and as a serving step chains them.

Tolerances, derived before the first run. A row that is stored as it is given is divided by a power of two, which is
exact, and rounded once: its bits are compared. A key after norm and rotation is the fp32 value of those (off by 32
fp32 roundings of sqrt(2) times the row's largest, as in test_paged_gpu.py) rounded to e4m3: half a step, 2^-4 of the
value or 2^(e - 10), with e the row's exponent. The attention reads the rows as they are held, so its tolerances are
those of test_paged_gpu.py with the dequantised rows, which are exact in bf16 and fp32.
"""
import math

import pytest
import torch

import paper_2609_03235_amd as sg
from test_paged_gpu import ATTN_CASES, ROPE_CASES, Case, _check_rounded, _i32, _plain_rope, _say

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
U8 = torch.uint8


def decoded(numbers, codes):
    """64-bit values of e4m3 numbers [..., d] and e8m0 codes [...], from their bits."""
    b = numbers.view(U8).long()
    exponent, mantissa = b >> 3 & 15, (b & 7).double()
    size = torch.where(exponent == 0, mantissa * 2.0 ** -9, (1 + mantissa / 8) * torch.exp2(exponent.double() - 7))
    size = torch.where(b & 0x7F == 0x7F, torch.full_like(size, math.nan), size)
    return torch.where(b > 127, -size, size) * torch.exp2(codes.view(U8).double() - 127).unsqueeze(-1)


def eight_bits(x):
    """The e4m3 bits and the code of rows [n, d], by whole steps in 64 bits."""
    x = x.double()
    fine = torch.isfinite(x)
    m, e = torch.frexp(torch.where(fine, x.abs(), torch.zeros_like(x)).amax(-1))
    e = torch.where(m == 0, -110, e.long() - 9 + (m > 0.875).long()).clamp(min=-110)
    y = torch.where(fine, x.abs() * torch.exp2(-e.double()).unsqueeze(-1), torch.zeros_like(x))
    _, k = torch.frexp(y)
    step = torch.exp2((k.long() - 1).clamp(min=-6).double() - 3)
    y = torch.round(y / step) * step  # half to even
    m, k = torch.frexp(y)
    bits = torch.where(y < 2.0 ** -6, y * 512, ((k.double() - 1 + 7) + (2 * m - 1)) * 8).long()
    bits = torch.where(fine, bits, torch.full_like(bits, 0x7F)) | torch.signbit(x).long() << 7
    return bits.to(U8), (e + 127).to(U8)


def same_numbers(got, want):
    nan = want & 0x7F == 0x7F
    return torch.equal(got & 0x7F == 0x7F, nan) and torch.equal(got[~nan], want[~nan])


def pool_of(n_pages, page, d, fill=0x7F, code=255):
    """A pool whose bytes are not numbers until something is stored."""
    b = lambda shape, x: torch.full(shape, x, dtype=U8, device=DEV)
    numbers = [b((n_pages, page, d), fill).view(torch.float8_e4m3fn) for _ in range(2)]
    return numbers + [b((n_pages, page), code).view(torch.float8_e8m0fnu) for _ in range(2)]


def rows_of(pool, slots, d):
    """Bits and codes of keys, and of values, in those slots."""
    flat = [p.view(U8).view(-1, d) if p.dim() == 3 else p.view(U8).view(-1) for p in pool]
    at = slots.long()
    return (flat[0][at], flat[2][at]), (flat[1][at], flat[3][at])


# ------------------------------------------------------------------ rows into pages
def _odd_rows(n, d, dtype, g):
    """Rows of every size: ordinary, of one value, zeros, next to every border of the power and of the rounding, the
    smallest and largest of the type, not finite."""
    x = torch.randn(n, d, generator=g, device=DEV)
    r = torch.arange(n, device=DEV)
    x = x * torch.exp2(((r * 37) % 250 - 125).float()).unsqueeze(-1)
    x[r % 11 == 3] = 0
    x[r % 13 == 5, 1:] = 0
    ties = torch.tensor([448.0, 17.0, 19.0, 21.0, 1.0625, 1.1875, 2.0 ** -10, 1.5 * 2.0 ** -9, 2.5 * 2.0 ** -9, -17.0,
                         -2.0 ** -10, -2.0 ** -7, 447.0, 240.0, 232.0, 0.0078125], device=DEV)
    some = r % 5 == 1
    x[some, :16] = ties
    x[some, 16:] = 0
    over = r % 17 == 4  # just past 448: the next power
    x[over] = 0
    x[over, 0] = 450.0
    x[over, 1:16] = ties[1:]
    x[r % 19 == 6, d - 1] = 3.3e38
    x[r % 23 == 7] = 1e-45
    x[r % 29 == 8, 3] = math.nan
    x[r % 31 == 9, 5] = math.inf
    x[r % 31 == 9, 6] = -math.inf
    x[r % 37 == 10] = math.nan
    x[r % 41 == 11, ::2] = -0.0
    return x.clamp(-3.38e38, 3.38e38).to(dtype) if dtype == BF else x


@pytest.mark.parametrize("dtype,d,n,page", [(BF, 128, 1, 16), (BF, 64, 777, 16), (F32, 128, 1000, 64), (F32, 64, 3, 32),
                                            (BF, 128, 4321, 128), (F32, 64, 513, 1024)])
def test_paged_store_fp8(dtype, d, n, page):
    _say(f"paged_store_fp8 {n} rows of {d} {dtype}")
    g = torch.Generator(device=DEV).manual_seed(n)
    k = _odd_rows(n, d, dtype, g)
    v = _odd_rows(n + 3, d, dtype, g)[3:].contiguous()
    n_pages = -(-n // page) + 2
    total = n_pages * page
    slots = torch.randperm(total, generator=g, device=DEV)[:n].to(torch.int32)
    slots[n // 2::7] = -1
    if n > 5:
        slots[1], slots[4] = total, 2**31 - 1
    pool = pool_of(n_pages, page, d, 0x3C, 9)
    sg.paged_store_fp8(k, v, slots, *pool)
    ok = (slots >= 0) & (slots < total)
    (kn, kc), (vn, vc) = rows_of(pool, slots[ok], d)
    for got, code, rows in ((kn, kc, k), (vn, vc, v)):
        want, wcode = eight_bits(rows[ok])
        assert torch.equal(code, wcode) and same_numbers(got, want)
    rest = torch.ones(total, dtype=torch.bool, device=DEV)
    rest[slots[ok].long()] = False
    for p in pool:
        assert (p.view(U8).flatten(0, 1)[rest] == (0x3C if p.dim() == 3 else 9)).all()


def test_paged_store_fp8_agrees_with_torchs_conversion():
    _say("paged_store_fp8 and torch's float8")
    x = torch.randn(500, 128, device=DEV)
    pool = pool_of(32, 16, 128)
    sg.paged_store_fp8(x, x, torch.arange(500, dtype=torch.int32, device=DEV), *pool)
    for pages, scales in ((pool[0], pool[2]), (pool[1], pool[3])):
        power = scales.float().view(-1)[:500, None]
        assert torch.equal((x / power).to(torch.float8_e4m3fn).view(U8), pages.view(-1, 128)[:500].view(U8))


def test_paged_store_fp8_of_nothing():
    pool = pool_of(2, 16, 64)
    none = torch.zeros(0, 64, device=DEV)
    sg.paged_store_fp8(none, none, _i32([]), *pool)
    assert all((p.view(U8) == (0x7F if p.dim() == 3 else 255)).all() for p in pool)


# ------------------------------------------------------------------ norm, rotation, store
def _check_bytes(numbers, codes, want, size, terms):
    """Rows of e4m3 bits and their codes against `want` (64 bits), computed with `terms` fp32 roundings of values up to
    `size` and rounded to 8 bits."""
    got = decoded(numbers, codes)
    e = codes.double() - 127
    err32 = terms * 2.0 ** -24 * size
    power = torch.exp2(e).unsqueeze(-1)
    top = want.abs().amax(-1, keepdim=True)
    # the power: the least that holds the row's largest, as far as fp32 tells
    assert (top <= 448 * power * (1 + 2.0 ** -22) + err32).all()
    assert ((top >= 224 * power * (1 - 2.0 ** -22) - err32) | (e.unsqueeze(-1) == -110)).all()
    tol = torch.maximum(2.0 ** -4 * (want.abs() + err32), 2.0 ** -10 * power) + err32
    err = (got - want).abs()
    assert torch.isfinite(got).all() and (err <= tol).all(), float((err / tol.clamp(min=1e-300)).max())


@pytest.mark.parametrize("T,hq,hkv,d,rot,norm,inter,dtype,first", ROPE_CASES)
@pytest.mark.parametrize("factor", [1.0, 1.34])
def test_norm_rope_store_fp8(T, hq, hkv, d, rot, norm, inter, dtype, first, factor):
    """The factor adds one rounding to each term of the rotation."""
    _say(f"norm_rope_fp8 {T} tokens {hq}/{hkv}/{d} rot {rot} {dtype} factor {factor}")
    g = torch.Generator(device=DEV).manual_seed(T + d)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)
    qkv = r(T, (hq + 2 * hkv) * d + 16).to(dtype)
    q, k, v = (x.view(T, -1, d) for x in qkv[:, :-16].split([hq * d, hkv * d, hkv * d], dim=1))
    page, pages = 16, -(-T * hkv // 16) + 2
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:T * hkv].to(torch.int32).view(T, hkv)
    slots[T // 2, 0] = -1
    slots[T // 3, hkv - 1] = pages * page
    pos = (first + torch.arange(T, device=DEV)).clamp(max=2**31 - 1).to(torch.int32)
    inv = (1e6 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / max(rot, 1))).float() if rot else None
    qw, kw = ((1 + 0.3 * r(d)).to(dtype) if norm else None for _ in range(2))
    pool = pool_of(pages, page, d, 0x3C, 9)
    out = sg.norm_rope_store_fp8(q, k, v, pos, slots, *pool, inv_freq=inv, q_weight=qw, k_weight=kw, eps=1e-6,
                                 interleaved=inter, rope_factor=factor)
    # the factor on the rotated columns of what the unscaled rotation gives
    scale = torch.ones(d, dtype=torch.float64, device=DEV)
    scale[:rot] = torch.tensor(factor, dtype=F32).double()
    wq = _plain_rope(q, qw, pos, inv, 1e-6, inter) * scale
    wk = _plain_rope(k, kw, pos, inv, 1e-6, inter) * scale
    big = lambda w: 2 ** 0.5 * w.abs().amax(-1, keepdim=True).clamp(min=1e-30)
    terms = 32 if (rot or norm) else 0
    _check_rounded(out, wq, big(wq), terms)
    ok = (slots >= 0) & (slots < pages * page)
    (kn, kc), (vn, vc) = rows_of(pool, slots[ok], d)
    _check_bytes(kn, kc, wk[ok], big(wk)[ok], terms)
    want, wcode = eight_bits(v[ok])
    assert torch.equal(vc, wcode) and torch.equal(vn, want)
    rest = torch.ones(pages * page, dtype=torch.bool, device=DEV)
    rest[slots[ok].long()] = False
    for p in pool:
        assert (p.view(U8).flatten(0, 1)[rest] == (0x3C if p.dim() == 3 else 9)).all()
    if factor == 1.0:  # the queries of the call over a pool of the rows' type, bit for bit
        kp, vp = (torch.zeros(pages, page, d, device=DEV, dtype=dtype) for _ in range(2))
        same = sg.norm_rope_store(q, k, v, pos, slots, kp, vp, inv_freq=inv, q_weight=qw, k_weight=kw, eps=1e-6,
                                  interleaved=inter)
        assert torch.equal(out, same)


def test_norm_rope_store_fp8_without_queries_in_place_and_of_nothing():
    _say("norm_rope_fp8 in place")
    T, hq, hkv, d = 50, 6, 2, 128
    g = torch.Generator(device=DEV).manual_seed(0)
    q, k, v = (torch.randn(T, h, d, generator=g, device=DEV).to(BF) for h in (hq, hkv, hkv))
    inv = (1e4 ** (-torch.arange(0, d, 2, device=DEV) / d)).float()
    pos = torch.arange(T, device=DEV, dtype=torch.int32)
    slots = torch.arange(T * hkv, device=DEV, dtype=torch.int32).view(T, hkv)
    a, b, c = (pool_of(8, 16, d) for _ in range(3))
    out = sg.norm_rope_store_fp8(q, k, v, pos, slots, *a, inv_freq=inv)
    q2 = q.clone()
    assert sg.norm_rope_store_fp8(q2, k, v, pos, slots, *b, inv_freq=inv, q_out=q2) is q2 and torch.equal(q2, out)
    assert sg.norm_rope_store_fp8(None, k, v, pos, slots, *c, inv_freq=inv) is None
    for x, y, z in zip(a, b, c):
        assert torch.equal(x.view(U8), y.view(U8)) and torch.equal(x.view(U8), z.view(U8))
    none = sg.norm_rope_store_fp8(q[:0], k[:0], v[:0], pos[:0], slots[:0], *c, inv_freq=inv)
    assert none.shape == (0, hq, d) and all(torch.equal(x.view(U8), z.view(U8)) for x, z in zip(a, c))


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 128), (F32, 64), (BF, 64)])
def test_norm_rope_store_fp8_copies_as_the_store(dtype, d):
    """Without norm and rotation keys too are the rows that paged_store_fp8 makes: every odd row bit for bit."""
    _say(f"norm_rope_fp8 as a copy {dtype} {d}")
    g = torch.Generator(device=DEV).manual_seed(3)
    T, hkv = 300, 3
    k, v = (_odd_rows(T * hkv, d, dtype, g).view(T, hkv, d) for _ in range(2))
    slots = torch.randperm(64 * 16, generator=g, device=DEV)[:T * hkv].to(torch.int32).view(T, hkv)
    a, b = pool_of(64, 16, d), pool_of(64, 16, d)
    sg.norm_rope_store_fp8(None, k, v, _i32([0] * T), slots, *a)
    sg.paged_store_fp8(k.view(-1, d), v.view(-1, d), slots.view(-1), *b)
    for x, y in zip(a, b):
        if x.dim() == 3:
            assert same_numbers(x.view(U8), y.view(U8))
        else:
            assert torch.equal(x.view(U8), y.view(U8))


# ------------------------------------------------------------------ attention
class Case8(Case):
    """A Case whose rows are in 8 bits; past the segments' rows the pool holds NaN and codes of 255."""

    def __init__(self, new, rows, hq, hkv, d, page, dtype, seed=0, pad=0, spread=1.0):
        super().__init__(new, rows, hq, hkv, d, page, dtype, seed=seed, pad=pad, spread=spread)
        g = torch.Generator(device=DEV).manual_seed(seed + 1)
        n_pages = self.k_pages.shape[0]
        self.pool = pool_of(n_pages, page, d)
        for s in range(len(rows)):
            for name, at in (("k", 0), ("v", 1)):
                x = getattr(self, name)[s]
                if name == "v":  # values of rows of different sizes, so that their powers differ
                    x = x.double() * torch.exp2(torch.randint(-3, 4, (x.shape[0], 1), generator=g, device=DEV).double())
                self.put(s, at, x)

    def slots(self, s):
        at = torch.arange(self.rows_host[s], device=DEV)
        return self.tables[s].long()[at // self.page] * self.page + at % self.page

    def put(self, s, at, x):
        """Rows x as segment s's keys (at 0) or values (1)."""
        bits, codes = eight_bits(x)
        slot = self.slots(s)
        self.pool[at].view(U8).view(-1, self.d)[slot] = bits
        self.pool[2 + at].view(U8).view(-1)[slot] = codes
        value = decoded(bits, codes).float()
        (self.k if at == 0 else self.v)[s] = value

    def call(self, max_new=None, **kw):
        return sg.paged_attention_fp8(self.q, *self.pool, self.tables, self.rows, self.cu, self.hkv,
                                      max_new=max_new or max(max(self.new), 1), **kw)


@pytest.mark.parametrize("case", ATTN_CASES)
@pytest.mark.parametrize("causal", [True, False])
def test_paged_attention_fp8(case, causal):
    new, rows, hq, hkv, d, page, dtype = case
    _say(f"paged_attention_fp8 new {new[:6]} rows {rows[:6]} {hq}/{hkv}/{d} page {page} {dtype} causal {causal}")
    c = Case8(new, rows, hq, hkv, d, page, dtype, seed=len(rows) + d, pad=3)
    for out_dtype in (BF, F32):
        out = torch.full((c.T, hq, d), 7.0, device=DEV, dtype=out_dtype)
        lse = torch.full((c.T, hq), 7.0, device=DEV)
        c.call(causal=causal, out=out, lse=lse, out_dtype=out_dtype)
        c.check(out, lse, causal)
        n = sum(new)
        assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()
        blind = torch.isinf(lse[:n])
        assert (out[:n][blind] == 0).all()


@pytest.mark.parametrize("new,rows,hq,hkv,dtype", [([1], [57000], 1, 1, BF), ([21], [57000], 1, 1, BF),
                                                   ([2, 1], [40000, 17, 3, 30000], 14, 2, F32),
                                                   ([300], [900, 901, 30000, 5], 16, 4, BF)])
def test_paged_attention_fp8_of_many_parts(new, rows, hq, hkv, dtype):
    _say(f"many parts {new} {rows}")
    c = Case8(new, rows, hq, hkv, 128, 64, dtype, seed=5)
    out, lse = c.call(out_dtype=F32)
    c.check(out, lse)
    again = c.call(out_dtype=F32)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("dtype,out_dtype,d", [(BF, BF, 128), (BF, F32, 64), (F32, F32, 64), (F32, BF, 128)])
def test_paged_attention_fp8_of_many_prompts(dtype, out_dtype, d):
    new = [40, 33, 0, 70, 5, 1] * 50
    rows = [n + (17 * i) % 150 for i, n in enumerate(x for n in new for x in (n, n))]
    _say(f"many prompts {dtype} -> {out_dtype} d {d}")
    c = Case8(new, rows, 16, 2, d, 32, dtype, seed=d)
    out, lse = c.call(out_dtype=out_dtype)
    c.check(out, lse)


@pytest.mark.parametrize("new", [[1], [30]])
@pytest.mark.parametrize("spread", [50.0, 0.0])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_paged_attention_fp8_far_logits(new, spread, dtype):
    _say(f"far logits {new} {spread} {dtype}")
    c = Case8(new, [3000, 2999], 14, 2, 128, 64, dtype, seed=9, spread=spread)
    for od in (BF, F32):
        out, lse = c.call(out_dtype=od)
        c.check(out, lse)


@pytest.mark.parametrize("n", [1, 5, 64])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_attention_of_logits_up_to_2_to_30(sign, dtype, d, n):
    """The largest logits that the contract takes, about 2^30 and -2^30, in pools of either kind. Two rows far from each
    other share the largest one, the others are smaller by 2^26 at least: the output is the mean of the two rows'
    values. The exponentials' arguments are off from what they would be by half a step of fp32 at such logits, up to
    2^6, but all by the same, so that the weights are 1/2 each, and the rest is a few roundings, 2^-21 of the values'
    sizes (fp32 output keeps the probabilities' bits)."""
    _say(f"large logits {sign} {dtype} d {d}, {n} tokens")
    L, page = 9000, 16
    g = torch.Generator(device=DEV).manual_seed(n + d)
    k, v = torch.zeros(L, d, device=DEV), torch.randn(L, d, generator=g, device=DEV).bfloat16().float()
    numbers = torch.tensor([1.0, 1.25, 1.5, 1.625, 1.75], device=DEV)  # of e4m3 and of bf16
    k[:, 3] = numbers[torch.randint(0, 5, (L,), generator=g, device=DEV)] - (3.0 if sign < 0 else 0.0)
    two = [77, 8001]
    k[two, 3] = 1.875 if sign > 0 else -1.0
    q = torch.zeros(n, 8, d, device=DEV)
    q[:, :, 3] = 2.0 ** 29
    pages = L // page + 1
    tables = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)[None]
    at = torch.arange(L, device=DEV)
    slots = (tables[0].long()[at // page] * page + at % page).to(torch.int32)
    pool8 = pool_of(pages, page, d)
    pool = [torch.zeros(pages, page, d, device=DEV, dtype=dtype) for _ in range(2)]
    sg.paged_store(k.to(dtype), v.to(dtype), slots, *pool)
    sg.paged_store_fp8(k.to(dtype), v.to(dtype), slots, *pool8)
    _, (bits, codes) = rows_of(pool8, slots, d)
    held = decoded(bits, codes)
    for call, p, values in ((sg.paged_attention, pool, v.double()), (sg.paged_attention_fp8, pool8, held)):
        out, lse = call(q.to(dtype), *p, tables, _i32([L]), _i32([0, n]), 1, max_new=n, causal=False, scale=1.0,
                        out_dtype=F32)
        want, size = values[two].mean(0), values[two].abs().sum(0)
        assert ((out.double() - want).abs() <= 2.0 ** -21 * size).all()
        top = float(k[two[0], 3]) * 2.0 ** 29
        assert ((lse.double() - top).abs() <= 2.0 ** -21 * abs(top)).all()


@pytest.mark.parametrize("new", [[1], [3], [40]])
@pytest.mark.parametrize("low,high", [(-124, -112), (-100, -70), (60, 90), (-40, 40)])
def test_paged_attention_fp8_powers(new, low, high):
    """Values whose rows' powers lie far from 1, and far from each other."""
    _say(f"powers {new} {low} to {high}")
    c = Case8(new, [900, 77], 8, 2, 64, 16, BF, seed=2)
    g = torch.Generator(device=DEV).manual_seed(low + 200)
    for s in range(2):
        n = c.rows_host[s]
        e = torch.randint(low, high, (n, 1), generator=g, device=DEV)
        c.put(s, 1, torch.randn(n, 64, generator=g, device=DEV).double() * torch.exp2(e.double()))
    out, lse = c.call(out_dtype=F32)
    c.check(out, lse)


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("G,n", [(1, 1), (8, 3), (8, 5), (1, 64), (8, 9)])
def test_paged_attention_fp8_of_one_row_of_every_code(dtype, d, G, n):
    """Segments of one row, with the codes 0 to 247, the keys' counted down: the last of a segment's n tokens sees the
    row, the ones before see nothing. Queries of zeros give it the probability 1 exactly, and the fp32 output is the
    row's values, bit for bit: numbers of 2^-6 to 240 are multiples of 2^-6, so that values are multiples of 2^-133,
    which bf16 holds, and below 2^128. Queries that undo their key's power give logits of ordinary size, of one product
    each: the log-sum-exp is off by a few fp32 roundings, 2^-21 of 1 and itself, and the output by 2^-21 of itself and
    2^-125."""
    _say(f"every code {dtype} d {d}, {G} heads, {n} tokens")
    g = torch.Generator(device=DEV).manual_seed(d + n)
    codes = torch.arange(248, device=DEV)
    bits = lambda: (torch.randint(4 << 3, 15 << 3, (248, d), generator=g, device=DEV)
                    | torch.randint(0, 2, (248, d), generator=g, device=DEV) << 7).to(U8)
    pool = pool_of(248, 16, d)  # segment s has page s; the bytes behind its row are no numbers
    key_codes = (247 - codes).clamp(min=3)
    pool[0].view(U8)[:, 0], pool[2].view(U8)[:, 0] = bits(), key_codes.to(U8)
    pool[1].view(U8)[:, 0], pool[3].view(U8)[:, 0] = bits(), codes.to(U8)
    k, v = decoded(pool[0][:, 0], pool[2][:, 0]), decoded(pool[1][:, 0], pool[3][:, 0])
    # two segments to a sequence; head i of a group looks at column 5 i + 1
    q = torch.zeros(124, n, 2, G, d, device=DEV)
    cols = (5 * torch.arange(G, device=DEV) + 1) % d
    undo = torch.exp2(127 - key_codes.double()).float()
    q[:, :, :, torch.arange(G, device=DEV), cols] = undo.view(124, 1, 2, 1).expand(124, n, 2, G)
    tables = codes.to(torch.int32)[:, None].contiguous()
    v = v.view(124, 2, 1, d).expand(124, 2, G, d)
    for x in (torch.zeros_like(q), q):
        out, lse = sg.paged_attention_fp8(x.view(124 * n, 2 * G, d).to(dtype), *pool, tables, _i32([1] * 248),
                                          _i32([i * n for i in range(125)]), 2, max_new=n, out_dtype=F32)
        out, lse = out.view(124, n, 2, G, d), lse.view(124, n, 2, G)
        assert (out[:, :-1] == 0).all() and (lse[:, :-1] == -math.inf).all()
        if x is q:
            want = (k[:, cols].view(124, 2, G) * undo.double().view(124, 2, 1)) / math.sqrt(d)
            assert ((lse[:, -1].double() - want).abs() <= 2.0 ** -21 * (1 + want.abs())).all()
            assert ((out[:, -1].double() - v).abs() <= 2.0 ** -21 * v.abs() + 2.0 ** -125).all()
        else:
            assert (lse[:, -1] == 0).all() and torch.equal(out[:, -1].double(), v)


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("n", [1, 64])
def test_paged_attention_fp8_of_the_largest_values(dtype, d, n):
    """Rows stored from the type's largest numbers: below 1.9375 * 2^127 they come back as the numbers that they were
    rounded to, from there on as infinities, each in its own column alone."""
    _say(f"largest values {dtype} d {d}, {n} tokens")
    border = 1.9375 * 2.0 ** 127
    v = torch.full((1, d), 3.0e38, device=DEV, dtype=F32)  # 225.7 * 2^120: held as 224
    v[0, 3], v[0, 4], v[0, 9] = border, -border, torch.finfo(dtype).max
    v[0, 7] = 1.9296875 * 2.0 ** 127  # 247 * 2^120, a number of bf16: held as 240
    v[0, 8] = -1.0
    v = v.to(dtype)
    pool = pool_of(1, 16, d)
    sg.paged_store_fp8(torch.zeros_like(v), v, _i32([0]), *pool)
    q = torch.zeros(n, 1, d, device=DEV, dtype=dtype)
    out, lse = sg.paged_attention_fp8(q, *pool, _i32([[0]]), _i32([1]), _i32([0, n]), 1, max_new=n, out_dtype=F32)
    want = torch.full((d,), 224 * 2.0 ** 120, device=DEV, dtype=torch.float64)
    want[7], want[8] = 240 * 2.0 ** 120, -0.0
    want[3], want[4], want[9] = math.inf, -math.inf, math.inf
    fine = torch.isfinite(want)
    assert torch.equal(out[-1, 0].double()[fine], want[fine]) and not torch.isfinite(out[-1, 0][~fine]).any()
    assert lse[-1, 0] == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new", [[1, 1], [20, 70]])
def test_paged_attention_fp8_scale_and_bounds(dtype, new):
    _say(f"scale {dtype} {new}")
    c = Case8(new, [90, 200, 300, 71], 6, 2, 64, 16, dtype, seed=4)
    for scale in (0.3, -0.11):
        out, none = c.call(max_new=max(new) + 500, scale=scale, with_lse=False)
        assert none is None
        c.check(out, None, scale=scale)


@pytest.mark.parametrize("new", [[1], [60]])
def test_paged_attention_fp8_bad_pages_read_as_zeros(new):
    _say(f"bad pages {new}")
    c = Case8(new, [500, 300], 8, 2, 128, 16, BF, seed=6)
    for s, j, bad in ((0, 3, -1), (0, 20, c.pool[0].shape[0]), (1, 0, 2**31 - 1), (1, 5, -2**31)):
        c.tables[s, j] = bad
        c.k[s][16 * j:16 * j + 16] = 0
        c.v[s][16 * j:16 * j + 16] = 0
    out, lse = c.call(out_dtype=F32)
    c.check(out, lse)


ODD_CASES = [
    (2, [5, 1], [70, 200, 33, 1000], BF),        # 5 query rows of 16
    (6, [6, 3], [9000, 61, 33, 1000], BF),       # 18 of 32, a segment cut into many parts
    (6, [16, 1], [130, 12000, 33, 40], BF),      # 48
    (8, [40, 33], [70, 9000, 33, 1000], BF),     # 128
    (2, [13, 1], [9000, 200, 33, 90], F32),      # 13 of 16
    (4, [15, 15], [70, 7000, 15, 16], F32),      # 30 of 32
    (8, [40, 33], [7000, 200, 40, 1000], F32),   # 128
]


@pytest.mark.parametrize("hq,new,rows,dtype", ODD_CASES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("byte", [0x7F, 0xFF])
def test_paged_attention_fp8_values_alone_that_are_not_finite(hq, new, rows, dtype, d, byte):
    """Not finite are the outputs of exactly the columns of NaN values of the tokens that see their rows; every other
    output, and every lse, is that of the clean run bit for bit."""
    _say(f"values {byte} {dtype} {new} over {rows} d {d}")
    c = Case8(new, rows, hq, 2, d, 16, dtype, seed=13)
    n, G = new[0], hq // 2
    for od in (BF, F32):
        clean, clean_lse = c.call(out_dtype=od)
        odd = torch.zeros(clean.shape, dtype=torch.bool, device=DEV)
        saved = c.pool[1].clone()
        for s, token, cols in ((0, n - 2, (5, 8)), (0, n - 1, (0, d - 1)), (1, n - 1, (6, 7)), (1, n - 2, (d - 2,))):
            slot = int(c.slots(s)[rows[s] - n + token])
            for col in cols:
                c.pool[1].view(U8).view(-1, d)[slot, col] = byte
                odd[token:n, s * G:(s + 1) * G, col] = True
        out, lse = c.call(out_dtype=od)
        assert torch.equal(lse, clean_lse)
        assert not torch.isfinite(out[odd]).any() and torch.equal(out[~odd], clean[~odd])
        c.pool[1] = saved


@pytest.mark.parametrize("hq,new,rows,dtype", ODD_CASES)
def test_paged_attention_fp8_rows_to_come(hq, new, rows, dtype):
    """NaN keys, and rows of code 255, reach no token that does not see them; those that do come out not finite."""
    _say(f"rows to come {dtype} {new} over {rows}")
    d = 128
    c = Case8(new, rows, hq, 2, d, 16, dtype, seed=13)
    n, G = new[0], hq // 2
    clean, clean_lse = c.call(out_dtype=F32)
    saved = [p.clone() for p in c.pool]
    for what in ("key", "key code", "value code"):
        slot = int(c.slots(0)[rows[0] - 2])  # the token before the last of the first sequence, its first KV head
        if what == "key":
            c.pool[0].view(U8).view(-1, d)[slot, 3] = 0x7F
        else:
            c.pool[2 if what == "key code" else 3].view(U8).view(-1)[slot] = 255
        out, lse = c.call(out_dtype=F32)
        odd = torch.zeros(c.T, c.hq, dtype=torch.bool, device=DEV)
        odd[n - 2:n, :G] = True
        assert torch.equal(out[~odd], clean[~odd]) and torch.equal(lse[~odd], clean_lse[~odd]), what
        assert not torch.isfinite(out[odd]).any(), what
        if what == "value code":
            assert torch.equal(lse, clean_lse)
        else:
            assert not torch.isfinite(lse[odd]).any()
        c.pool = [p.clone() for p in saved]


@pytest.mark.parametrize("hq,new,rows,dtype", ODD_CASES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", ["key", "key code", "value code"])
def test_paged_attention_fp8_nan_rows_within_a_segment(hq, new, rows, dtype, d, what):
    """A NaN key in the first or the last column, or a code of 255, among the rows that all tokens see and on the row
    of the last but one, in two segments: every instance, both types of output. Tokens and heads that do not see them
    come out as ever; keys that are NaN reach the log-sum-exp too, values do not."""
    _say(f"NaN rows: {what} {dtype} {new} over {rows} d {d}")
    c = Case8(new, rows, hq, 2, d, 16, dtype, seed=23)
    G, t0 = hq // 2, new[0]
    for od in (BF, F32):
        clean, clean_lse = c.call(out_dtype=od)
        saved = [p.clone() for p in c.pool]
        odd = torch.zeros(c.T, c.hq, dtype=torch.bool, device=DEV)
        for s, row, col in ((0, rows[0] - 2, 0), (3, (rows[3] - new[1]) // 2, d - 1)):
            slot = int(c.slots(s)[row])
            if what == "key":
                c.pool[0].view(U8).view(-1, d)[slot, col] = 0xFF
            else:
                c.pool[2 if what == "key code" else 3].view(U8).view(-1)[slot] = 255
            b, h = divmod(s, 2)
            first, n = t0 * b, new[b]
            sees = torch.arange(n, device=DEV) >= row - (rows[s] - n)
            odd[first:first + n, h * G:(h + 1) * G] |= sees[:, None]
        assert odd.any() and not odd.all()
        out, lse = c.call(out_dtype=od)
        c.check(torch.where(odd[..., None], clean, out), torch.where(odd, clean_lse, lse))
        assert not torch.isfinite(out[odd]).any()
        if what == "value code":
            assert torch.equal(lse, clean_lse)
        else:
            assert not torch.isfinite(lse[odd]).any()
        c.pool = saved


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("hq,new", [(2, [1]), (8, [5]), (8, [11]), (8, [40])])
@pytest.mark.parametrize("low,high", [(-112, -100), (-100, -60), (60, 90), (-40, 40)])
def test_paged_attention_fp8_spread_powers(hq, new, dtype, d, low, high):
    """Values whose rows' powers lie far from 1, and far from each other, in tiles of one, two and three blocks and of
    many rows, for both types of output. (Rows no smaller than the stores write: at 2^-110 the probabilities' last bits
    are bf16's smallest subnormals.)"""
    _say(f"spread powers {dtype} d {d} {new} {low} to {high}")
    c = Case8(new, [900, 77], hq, 2, d, 16, dtype, seed=3)
    g = torch.Generator(device=DEV).manual_seed(low + 300)
    for s in range(2):
        n = c.rows_host[s]
        e = torch.randint(low, high, (n, 1), generator=g, device=DEV)
        c.put(s, 1, torch.randn(n, d, generator=g, device=DEV).double() * torch.exp2(e.double()))
    for od in (BF, F32):
        out, lse = c.call(out_dtype=od)
        c.check(out, lse)


def test_paged_attention_fp8_cuts_lengths_to_the_buffers():
    _say("cut lengths")
    c = Case8([5], [64, 64], 4, 2, 64, 16, BF, seed=8)
    c.tables = c.tables[:, :4].contiguous()
    c.rows.fill_(2**31 - 1)
    c.cu.copy_(_i32([-4, 5]))
    out, lse = c.call()
    c.check(out, lse)
    c.cu.copy_(_i32([0, 2**30]))
    out2, _ = c.call()
    assert torch.equal(out, out2)
    for max_new in (2, 3):
        kept = torch.full_like(out, 3.0)
        lse2 = torch.full_like(lse, 3.0)
        c.call(max_new=max_new, out=kept, lse=lse2)
        assert (kept[max_new:] == 3.0).all() and (lse2[max_new:] == 3.0).all()
        c.check(kept, lse2, only=torch.arange(5, device=DEV) < max_new)


def test_paged_attention_fp8_of_nothing():
    c = Case8([0, 0], [5, 0], 2, 1, 64, 16, BF)
    out, lse = c.call(max_new=4)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)


@pytest.mark.parametrize("hq,new", [(2, [3]), (4, [40])])
def test_paged_attention_fp8_of_many_segments(hq, new):
    _say(f"many segments {new}")
    n = [1 if i % 7 else 0 for i in range(600)]
    n[300] = new[0]
    c = Case8(n, [(i * 53) % 70 + n[i // 2] for i in range(1200)], hq, 2, 64, 16, BF, seed=61)
    out, lse = c.call(out_dtype=F32)
    c.check(out, lse)


@pytest.mark.parametrize("new,rows,hq,hkv,d", [
    ([1, 1], [700, 30000, 1, 64], 16, 2, 128),          # 8 rows of 16
    ([1, 2, 1], [90, 4000, 333], 16, 1, 64),            # 32 rows
    ([6, 1, 3], [5000, 129, 7, 700, 16, 90], 16, 2, 128),  # 48 rows
])
def test_paged_attention_fp8_of_few_rows_keeps_the_probabilities_bits(new, rows, hq, hkv, d):
    """Up to 48 query rows per KV head probabilities go in as bf16 terms: three for fp32 output, all their bits, and two
    for bf16 output, off by 2^-16 of a probability at most: bf16 has 8 significant bits, 2^-7 from 1 to the next number,
    so the first term leaves at most half of that, 2^-8 of the probability, and the second 2^-8 of what is left. So
    bf16 output is within 2^-16 A and half a step of its own, 2^-8 of the value, of the 64-bit value, beside what the
    fp32 output is off by."""
    _say(f"probabilities {new} {hq}/{hkv}/{d}")
    c = Case8(new, rows, hq, hkv, d, 16, BF, seed=17)
    out, lse = c.call(out_dtype=BF)
    fine, lse2 = c.call(out_dtype=F32)
    c.check(fine, lse2)
    assert torch.equal(lse, lse2)
    want, _, A, big, seen, scale = c.want()
    delta = 2.0 ** -21 * scale * big + 2.0 ** -22 * (1 + scale * big)
    off = (2 * delta + 2.0 ** -16 + (seen / 4 + 64) * 2.0 ** -24)[..., None] * A
    err = (out.double() - want).abs()
    assert (err <= off + 2.0 ** -8 * (want.abs() + off) * (1 + 2.0 ** -8)).all()


def test_paged_attention_fp8_pools_beyond_4_gib():
    """Pages whose bytes lie past 2^32 of the pool: stores, rotation and both attention kernels."""
    _say("8-bit pools beyond 4 GiB")
    d, page, hq, hkv = 128, 256, 8, 2
    n_pages = (5 << 30) // (page * d)
    pool = pool_of(n_pages, page, d)
    for new in ([1, 2], [40, 9]):
        c = Case8(new, [300, 700, 257, 512], hq, hkv, d, page, BF, seed=21)
        far = c.tables.clone()
        used = c.tables >= 0
        far[used] = n_pages - 1 - c.tables[used]
        c.tables = far
        for s in range(4):
            slot = c.slots(s)
            sg.paged_store_fp8(c.k[s].to(BF), c.v[s].to(BF), slot.to(torch.int32), *pool)
            (kn, kc), (vn, vc) = rows_of(pool, slot, d)
            assert torch.equal(decoded(kn, kc).float(), c.k[s]) and torch.equal(decoded(vn, vc).float(), c.v[s])
        c.pool = pool
        out, lse = c.call(out_dtype=F32)
        c.check(out, lse)
    k = torch.randn(3, hkv, d, device=DEV).to(BF)
    slots = (n_pages * page - 1 - torch.arange(6, device=DEV)).to(torch.int32).view(3, hkv)
    sg.norm_rope_store_fp8(None, k, k, _i32([0, 0, 0]), slots, *pool)
    want, code = eight_bits(k.view(-1, d))
    (kn, kc), _ = rows_of(pool, slots.flatten(), d)
    assert torch.equal(kn, want) and torch.equal(kc, code)


# ------------------------------------------------------------------ together
def _serve_state(B, hkv, page, max_pages, n_pages, d):
    return dict(rows=torch.zeros(B * hkv, dtype=torch.int32, device=DEV), head=_i32([0]),
                tables=torch.full((B * hkv, max_pages), -1, dtype=torch.int32, device=DEV),
                free=torch.randperm(n_pages, device=DEV).to(torch.int32), pool=pool_of(n_pages, page, d))


def _segment(st, s, n, page, d):
    at = torch.arange(n, device=DEV)
    slot = st["tables"][s].long()[at // page] * page + at % page
    return rows_of(st["pool"], slot, d)


@pytest.mark.parametrize("chunks", [[5, 1, 1], [70, 3, 40]])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_fp8_steps_against_64_bits(chunks, dtype):
    """A compressed prompt's rows into pages, then steps of page_update, norm_rope_store_fp8 and paged_attention_fp8,
    each against 64 bits; the rows come out the same however the tokens are cut into steps."""
    _say(f"8-bit steps {chunks} {dtype}")
    B, hq, hkv, d, page, C = 3, 8, 2, 64, 16, 600
    g = torch.Generator(device=DEV).manual_seed(7)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV).to(dtype)
    budgets = [200, 77]
    res = sg.compress_layer(r(B, hq, 16, d), r(B, hkv, C, d), r(B, hkv, C, d), budgets, pool_kernel=5, b_sink=4,
                            b_window=32)
    n = sum(chunks)
    q, k, v = (r(B, n, h, d) for h in (hq, hkv, hkv))
    inv = (1e4 ** (-torch.arange(0, d, 2, device=DEV) / d)).float()
    wts = [(1 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(dtype) for _ in range(2)]
    pos = C + torch.arange(n, device=DEV, dtype=torch.int32)
    wk = torch.stack([_plain_rope(k[b], wts[1], pos, inv, 1e-6, False) for b in range(B)])
    big = lambda w: 2 ** 0.5 * w.abs().amax(-1, keepdim=True)
    ends = []
    for plan in (chunks, [n]):
        st = _serve_state(B, hkv, page, 32, 200, d)
        up = sg.page_update(st["rows"], _i32(budgets * B), st["tables"], st["free"], st["head"], page_size=page,
                            n_slots=sum(budgets) * B, by_segment=True, rows_out=st["rows"], head_out=st["head"])
        sg.paged_store_fp8(res["k_c"], res["v_c"], up["slots"], *st["pool"])
        done = 0
        for m in plan:
            up = sg.page_update(st["rows"], _i32([m] * B), st["tables"], st["free"], st["head"], page_size=page,
                                n_slots=B * m, rows_out=st["rows"], head_out=st["head"])
            cut = lambda x: x[:, done:done + m].reshape(B * m, -1, d)
            qr = sg.norm_rope_store_fp8(cut(q), cut(k), cut(v), pos[done:done + m].repeat(B), up["slots"],
                                        *st["pool"], inv_freq=inv, q_weight=wts[0], k_weight=wts[1])
            out, lse = sg.paged_attention_fp8(qr, *st["pool"], st["tables"], up["rows"], up["cu"], hkv, max_new=m)
            done += m
            c = Case.__new__(Case)
            c.new, c.hq, c.hkv, c.d, c.T, c.q, c.k, c.v = [m] * B, hq, hkv, d, B * m, qr, [], []
            c.rows_host = [budgets[s % hkv] + done for s in range(B * hkv)]
            for s in range(B * hkv):
                (kn, kc), (vn, vc) = _segment(st, s, c.rows_host[s], page, d)
                c.k.append(decoded(kn, kc))
                c.v.append(decoded(vn, vc))
                b, h = divmod(s, hkv)
                lo = int(res["offsets"][s])
                for bits, codes, old, new in ((kn, kc, res["k_c"], None), (vn, vc, res["v_c"], v[b, :done, h])):
                    want, code = eight_bits(old[lo:lo + budgets[h]])
                    assert torch.equal(bits[:budgets[h]], want) and torch.equal(codes[:budgets[h]], code)
                    if new is not None:
                        want, code = eight_bits(new)
                        assert torch.equal(bits[budgets[h]:], want) and torch.equal(codes[budgets[h]:], code)
                _check_bytes(kn[budgets[h]:], kc[budgets[h]:], wk[b, :done, h], big(wk[b, :done, h]), 32)
            c.check(out, lse)
        ends.append([_segment(st, s, budgets[s % hkv] + n, page, d) for s in range(B * hkv)])
    for a, b in zip(*ends):
        for x, y in zip(a, b):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


def test_fp8_captured_steps_replay_with_new_lengths():
    """One captured step replayed while the cache grows and shrinks, against eager steps on a second cache, with eager
    work between the replays."""
    _say("captured 8-bit steps")
    B, hq, hkv, d, page, T = 4, 14, 2, 128, 16, 8
    g = torch.Generator(device=DEV).manual_seed(5)
    inv = (1e6 ** (-torch.arange(0, d, 2, device=DEV) / d)).float()
    a, b = (_serve_state(B, hkv, page, 64, 600, d) for _ in range(2))
    b["free"].copy_(a["free"])
    io = dict(q=torch.zeros(T, hq, d, device=DEV, dtype=BF), k=torch.zeros(T, hkv, d, device=DEV, dtype=BF),
              v=torch.zeros(T, hkv, d, device=DEV, dtype=BF), pos=_i32([0] * T), add=_i32([0] * B))
    ws = sg.alloc_workspace(sg.paged_attention_fp8_workspace_size(io["q"], hkv, B, max_new=T), DEV)

    def step(st, ws):
        up = sg.page_update(st["rows"], io["add"], st["tables"], st["free"], st["head"], page_size=page, n_slots=T,
                            rows_out=st["rows"], head_out=st["head"])
        qr = sg.norm_rope_store_fp8(io["q"], io["k"], io["v"], io["pos"], up["slots"], *st["pool"], inv_freq=inv)
        out = torch.zeros(T, hq, d, device=DEV, dtype=BF)
        lse = torch.zeros(T, hq, device=DEV)
        return sg.paged_attention_fp8(qr, *st["pool"], st["tables"], up["rows"], up["cu"], hkv, max_new=T, out=out,
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
        for x, y in zip(a["pool"], b["pool"]):
            assert torch.equal(x.view(U8), y.view(U8))


def test_fp8_calls_on_another_stream():
    _say("another stream")
    c = Case8([40, 1], [500, 40, 300, 77], 14, 2, 128, 16, BF, seed=12)
    want, want_lse = c.call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, lse = c.call(stream=side)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    out, _ = c.call(stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(out, want)
    x = torch.randn(70, 64, device=DEV)
    slots = torch.arange(70, dtype=torch.int32, device=DEV)
    a, b, d = (pool_of(6, 16, 64) for _ in range(3))
    torch.cuda.synchronize()
    sg.paged_store_fp8(x, x, slots, *a)
    sg.paged_store_fp8(x, x, slots, *b, stream=side)
    q = sg.norm_rope_store_fp8(x[:, None], x[:, None], x[:, None], slots, slots[:, None].contiguous(), *d, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(q, x[:, None])
    for y, z, w in zip(a, b, d):
        assert torch.equal(y.view(U8), z.view(U8)) and torch.equal(y.view(U8), w.view(U8))


def test_two_fp8_calls_at_once():
    _say("two at once")
    cases = [Case8([1, 1], [30000, 20000, 3000, 50], 14, 2, 128, 64, BF, seed=31),
             Case8([300, 77], [3000, 5000, 300, 77], 14, 2, 128, 16, BF, seed=32)]
    want = [c.call() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    ws = [sg.alloc_workspace(sg.paged_attention_fp8_workspace_size(c.q, c.hkv, 2, max_new=max(c.new)), DEV)
          for c in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        got = [c.call(workspace=w, stream=s) for c, w, s in zip(cases, ws, streams)]
        torch.cuda.synchronize()
        for (o, l), (wo, wl) in zip(got, want):
            assert torch.equal(o, wo) and torch.equal(l, wl)


def test_two_captured_fp8_calls_share_a_workspace():
    _say("two graphs, one workspace")
    cases = [Case8([1, 1], [9000, 20000, 3000, 50], 14, 2, 128, 64, BF, seed=41),
             Case8([130, 7], [3000, 500, 300, 77], 14, 2, 128, 16, BF, seed=42)]
    want = [c.call() for c in cases]
    ws = sg.alloc_workspace(max(sg.paged_attention_fp8_workspace_size(c.q, c.hkv, 2, max_new=max(c.new))
                                for c in cases), DEV)
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


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new", [[1], [20], [70]])
def test_fp8_table_of_repeated_pages_past_2_to_25_rows(new, dtype):
    """A segment of 40 million rows whose table names the same 64 pages over and over: its softmax is that of the
    pages' rows, each many times, so out is that of one round of them and lse larger by the log of the rounds. A worker
    adds 79000 rows, 16 or more at a time per lane group and product: 2500 roundings at most meet in a sum."""
    _say(f"long table {new} {dtype}")
    d, page, P, rounds = 64, 1024, 64, 620
    g = torch.Generator(device=DEV).manual_seed(0)
    pool = pool_of(P, page, d)
    k, v = (torch.randn(P * page, d, generator=g, device=DEV) for _ in range(2))
    sg.paged_store_fp8(k, v, torch.arange(P * page, dtype=torch.int32, device=DEV), *pool)
    kd, vd = decoded(pool[0], pool[2]).view(-1, d), decoded(pool[1], pool[3]).view(-1, d)
    tables = torch.arange(P, dtype=torch.int32, device=DEV).repeat(rounds)[None].contiguous()
    q = torch.randn(sum(new), 4, d, generator=g, device=DEV).to(dtype)
    out, lse = sg.paged_attention_fp8(q, *pool, tables, _i32([P * page * rounds]), _i32([0, len(q)]), 1,
                                      max_new=max(new), causal=False, out_dtype=F32)
    y = q.double().flatten(0, 1) @ kd.T / 8
    want, wlse = torch.softmax(y, 1) @ vd, torch.logsumexp(y, 1) + math.log(rounds)
    assert (out.double().flatten(0, 1) - want).abs().max() < 2500 * 2.0 ** -24 + 2e-5
    assert (lse.double().flatten() - wlse).abs().max() < 2500 * 2.0 ** -24 + 2e-5


def test_fp8_shared_pages_and_padding():
    """Two sequences whose tables name the same pages read the same rows; tokens behind the last sequence's keep what
    out and lse held."""
    _say("shared pages")
    c = Case8([1, 3], [500, 90, 500, 90], 8, 2, 128, 16, BF, seed=51, pad=5)
    c.tables[2:] = c.tables[:2]
    c.k[2:], c.v[2:] = c.k[:2], c.v[:2]
    out, lse = torch.full((c.T, 8, 128), 9.0, device=DEV), torch.full((c.T, 8), 9.0, device=DEV)
    c.call(out_dtype=F32, out=out, lse=lse)
    c.check(out, lse)
    assert (out[4:] == 9.0).all() and (lse[4:] == 9.0).all()


def test_norm_rope_store_fp8_of_more_tokens_than_a_launch_holds():
    """2^26 + 37 tokens, a wave each, go in several launches; tokens around each power of two from 2^24 on are
    compared, and the slots of the others are -1."""
    _say("norm_rope_fp8 of 2^26 + 37 tokens")
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
    a, b = pool_of(1, 16, d), pool_of(1, 16, d)
    out = sg.norm_rope_store_fp8(k, k, k, pos, slots, *a, inv_freq=inv)
    want = sg.norm_rope_store_fp8(k[some], k[some], k[some], pos[some], slots[some], *b, inv_freq=inv)
    assert torch.equal(out[some], want)
    for x, y in zip(a, b):
        assert torch.equal(x.view(U8), y.view(U8))
    rows = _plain_rope(k[some], None, pos[some], inv, 0.0, False)
    (kn, kc), _ = rows_of(b, slots[some, 0], d)
    _check_bytes(kn, kc, rows[:, 0], 2 ** 0.5 * rows[:, 0].abs().amax(-1, keepdim=True), 32)
