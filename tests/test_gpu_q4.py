"""A cache held in four bits: rows filed and read, exactly, and phase 2 over it, against 64 bits (oracle/star_q4.py).

Bounds.  Four-bit values are exact in the products.  A logit is a sum of d products held in 32 bits, and its argument of the
exponential two roundings more: off by (d + 4) 2^-24 of sum |q k| scale, at most.  Weights are rounded to half a step of bf16 (2^-8) at most, of
two parts (2^-16) or of fp32 (2^-24); their sums over n keys round n / 32 + 64 times.  A relative error of every weight
moves an output by that times sum p |v|, twice, because the sum of the weights has it too.
fp16 has a least step, 2^-24, and a row's largest weight is 2^10 or more when it is taken (2^(TOP + 1 - 4) to half of that in the row-tiled
kernel, 2^13.5 in the other): a weight may be off by half that step, 2^-25 / 2^10 of the largest, which is no more than the sum by which
outputs are divided.  Over all keys that is 2^-35 sum |v| at most.  (Keys whose values fp16 does not hold are weighted in bf16.)"""
import math

import pytest
import torch

import paper_2411_17116_amd as sa
from oracle import star_q4

pytestmark = pytest.mark.gpu


def _randn(gen, dtype, *size):
    return torch.randn(size, generator=gen).to(torch.float32 if dtype == "fp32" else torch.bfloat16).cuda()


def _bound(dtype, d, n, size, weights, total, parts):
    """Of an output whose rows have `size` = sum |q k| scale, `weights` = sum p |v| and `total` = sum |v|."""
    u = 2.0 ** -24
    step = u if dtype == "fp32" else 2.0 ** -16 if parts == 2 else 2.0 ** -8
    return weights * (step + 2 * u * ((d + 4) * size[:, None] + n / 32 + 64)) + total * 2.0 ** -35 + 1e-30


class Call:
    """A call's tensors, its cache filled by the oracle's quantiser with NaN behind the rows that hold something."""

    def __init__(self, dtype, B, Hq, Hkv, d, L, q, seed=0, block=None, spare=70, cached=None):
        gen = torch.Generator().manual_seed(seed + L + q)
        self.cached = L if cached is None else cached
        cap = self.cached + q + spare
        self.dtype, self.dims, self.q = dtype, (B, Hq, Hkv, d), q
        self.shape = sa.StarShape.make(dtype, B, Hq, Hkv, d, L, block or L, 0, cap)
        self.Q, self.K, self.V = (_randn(gen, dtype, B, q, H, d) for H in (Hq, Hkv, Hkv))
        self.cache = sa.alloc_q4_cache(self.shape)
        rows = slice(0, self.cached)
        for codes, scales in ((self.cache.k_codes, self.cache.k_scales), (self.cache.v_codes, self.cache.v_scales)):
            scales.fill_(255)
            codes.fill_(0x5a)
            codes[:, :, rows], scales[:, :, rows] = star_q4.quantise(_randn(gen, dtype, B, Hkv, self.cached, d))
        self.O = torch.full_like(self.Q, math.nan)
        self.ws = sa.alloc_q4_workspace(self.shape, q)
        self.scale = 1 / math.sqrt(d)

    def tensors(self):
        return self.cache.k_codes, self.cache.k_scales, self.cache.v_codes, self.cache.v_scales

    def appended(self):
        """The cache with the new rows filed, by the oracle."""
        out = [t.clone() for t in self.tensors()]
        for i, x in enumerate((self.K, self.V)):
            codes, scales = star_q4.quantise(x.transpose(1, 2))
            out[2 * i][:, :, self.cached:self.cached + self.q], out[2 * i + 1][:, :, self.cached:self.cached + self.q] = codes, scales
        return out

    def exact(self, tensors, b, h, append=True, lo=0, hi=None):
        g = h // (self.dims[1] // self.dims[2])
        n = self.cached + (self.q if append else 0)
        K, V = (star_q4.values(tensors[i][b, g, :n], tensors[i + 1][b, g, :n]) for i in (0, 2))
        return star_q4.attend(self.Q[b, :, h], K, V, self.scale, self.cached if append else None, lo, hi)

    def heads(self, few=4):
        B, Hq = self.dims[:2]
        every = [(b, h) for b in range(B) for h in range(Hq)]
        return every if len(every) <= few else [every[i * (len(every) - 1) // (few - 1)] for i in range(few)]

    def near(self, got, want, bound, what):
        got = got.double()
        assert got.shape == want.shape
        assert torch.equal(got.isnan(), want.isnan()), what
        off = (got - want).abs().nan_to_num(0.0)
        assert (off <= bound.nan_to_num(1.0)).all(), (what, off.max().item(), (off / bound).nan_to_num(0.0).max().item())

    def check_O(self, tensors, few=4):
        for b, h in self.heads(few):
            A, lse, weights, size, total = self.exact(tensors, b, h)
            bound = _bound(self.dtype, self.dims[3], self.cached + self.q, size, weights, total, 1)
            self.near(self.O[b, :, h], A, bound + A.abs() * (2.0 ** -24 if self.dtype == "fp32" else 2.0 ** -8), (b, h))

    def check_pair(self, tensors, A, LSE, append, few=4, lo=0, hi=None):
        for b, h in self.heads(few):
            want, lse, weights, size, total = self.exact(tensors, b, h, append, lo, hi)
            n = self.cached + self.q
            empty = lse == -math.inf
            assert torch.equal(LSE[b, h] == -math.inf, empty) and (A[b, h][empty] == 0).all()
            seen = ~empty
            if not seen.any():
                continue
            self.near(A[b, h][seen], want[seen], (_bound(self.dtype, self.dims[3], n, size, weights, total, 2) + want.abs() * 2.0 ** -24)[seen], (b, h))
            self.near(LSE[b, h][seen], lse[seen], (2.0 ** -24 * (2 * (self.dims[3] + 4) * size + n / 32 + 64 + 8 * lse.abs()))[seen], (b, h, "lse"))


# ------------------------------------------------------------------ rows


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64), ("fp32", 128)])
def test_every_bf16_value(dtype, d):
    """All 65536 bit patterns, with each exponent as the group's largest and with their neighbours."""
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    rows = [every.view(-1, d)]
    gen = torch.Generator().manual_seed(5)
    every = every[torch.isfinite(every)]
    for shift in (0, 1, 2, 3, 4, 30):       # elements next to a group's largest, smaller by up to that many powers of two
        x = every[torch.randperm(every.numel(), generator=gen)][: every.numel() // d * d].view(-1, d)
        lead = x[:, ::32].abs().clamp(min=1e-30)
        y = lead.repeat_interleave(32, 1) * torch.exp2(-torch.rand(x.shape, generator=gen) * shift) * torch.sign(x + 1e-45)
        y[:, ::32] = x[:, ::32]
        rows.append(y)
    x = torch.cat(rows).to(dt)
    grid = star_q4.GRID.float()
    ties = torch.stack([torch.cat([(grid[:-1] + grid[1:]) / 2, grid, -grid, -(grid[:-1] + grid[1:]) / 2, torch.tensor([6.0, 5.5])])] * 64)
    ties = ties * torch.exp2(torch.arange(64.0) - 31)[:, None]                  # 32 elements: every tie, at 64 sizes
    x = torch.cat([x, ties.view(-1, d).to(dt)]).cuda()
    n = x.shape[0]
    shape = sa.StarShape.make(dtype, 1, 1, 1, d, n, n, 0, n)
    cache = sa.alloc_q4_cache(shape)
    K = x.view(1, 1, n, d)
    V = K.flip(2).contiguous()
    sa.q4_store(shape, 0, n, K, V, cache)
    Ko, Vo = torch.empty_like(K), torch.empty_like(V)
    sa.q4_load(shape, 0, n, cache, Ko, Vo)
    torch.cuda.synchronize()
    for y, codes, scales, back in ((K, cache.k_codes, cache.k_scales, Ko), (V, cache.v_codes, cache.v_scales, Vo)):
        c, e = star_q4.quantise(y.cpu())
        assert torch.equal(scales.cpu(), e)
        assert torch.equal(codes.cpu(), c)
        want = star_q4.values(c, e)
        assert torch.equal(back.cpu().double().nan_to_num(9e99), want.nan_to_num(9e99))


def test_every_code_and_unit_reads_as_what_it_stands_for():
    n = 256
    shape = sa.StarShape.make("fp32", 1, 1, 1, 64, n, n, 0, n)
    cache = sa.alloc_q4_cache(shape)
    cache.k_codes[:] = torch.arange(256, dtype=torch.uint8).cuda().view(4, 64)[:, :32].repeat(64, 1)
    cache.v_codes[:] = torch.arange(256, dtype=torch.uint8).cuda().view(4, 64)[:, 32:].repeat(64, 1)
    unit = torch.arange(256).clamp(2, 252)
    unit[255] = 255
    cache.k_scales[:] = unit.to(torch.uint8).cuda()[:, None]
    cache.v_scales[:] = unit.flip(0).to(torch.uint8).cuda()[:, None]
    K, V = torch.zeros(1, 1, n, 64).cuda(), torch.zeros(1, 1, n, 64).cuda()
    sa.q4_load(shape, 0, n, cache, K, V)
    torch.cuda.synchronize()
    for x, c, e in ((K, cache.k_codes, cache.k_scales), (V, cache.v_codes, cache.v_scales)):
        assert torch.equal(x.double().nan_to_num(9e99), star_q4.values(c, e).nan_to_num(9e99))


@pytest.mark.parametrize("dtype,B,Hkv,d,cap,first,n,rows,plain", [
    ("bf16", 1, 1, 128, 1, 0, 1, 1, 0), ("bf16", 2, 3, 128, 50, 7, 33, 40, 5), ("fp32", 2, 3, 64, 50, 49, 1, 3, 2),
    ("fp32", 3, 1, 128, 17, 0, 17, 17, 0), ("bf16", 1, 8, 128, 5000, 1234, 3333, 4000, 600)])
def test_rows_of_their_numbers_and_no_others(dtype, B, Hkv, d, cap, first, n, rows, plain):
    gen = torch.Generator().manual_seed(cap + n)
    shape = sa.StarShape.make(dtype, B, Hkv, Hkv, d, 1, 1, 0, cap)
    K, V = _randn(gen, dtype, B, Hkv, rows, d), _randn(gen, dtype, B, Hkv, rows, d)
    cache = sa.alloc_q4_cache(shape)
    every = (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)
    for t in every:
        t.fill_(0xa5)
    want = [t.clone() for t in every]
    for i, x in enumerate((K, V)):
        want[2 * i][:, :, first:first + n], want[2 * i + 1][:, :, first:first + n] = star_q4.quantise(x[:, :, plain:plain + n])
    sa.q4_store(shape, first, n, K, V, cache, plain_row=plain)
    Ko, Vo = torch.full_like(K, 7.0), torch.full_like(V, 7.0)
    sa.q4_load(shape, first, n, cache, Ko, Vo, plain_row=plain)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(every, want))
    for i, x in enumerate((Ko, Vo)):
        assert torch.equal(x[:, :, plain:plain + n].double(), star_q4.values(want[2 * i][:, :, first:first + n], want[2 * i + 1][:, :, first:first + n]))
        x[:, :, plain:plain + n] = 7.0
        assert (x == 7.0).all()


# ------------------------------------------------------------------ attention

CALLS = [
    # one token: a single cached row, around units and splits, odd groups, several sequences
    ("bf16", 1, 1, 1, 128, 1, 1), ("bf16", 1, 4, 4, 128, 30, 1), ("bf16", 1, 32, 8, 128, 31, 1), ("bf16", 2, 10, 2, 128, 32, 1),
    ("bf16", 1, 8, 2, 128, 127, 1), ("bf16", 1, 8, 2, 128, 128, 1), ("bf16", 3, 6, 2, 128, 129, 1), ("bf16", 1, 32, 8, 128, 2000, 1),
    ("bf16", 4, 64, 8, 128, 4099, 1), ("bf16", 1, 16, 1, 128, 16385, 1), ("bf16", 1, 32, 8, 128, 70001, 1), ("bf16", 40, 8, 8, 128, 333, 1),
    # rows that fill 16, pass it, fill more
    ("bf16", 1, 8, 2, 128, 500, 4), ("bf16", 1, 8, 2, 128, 500, 5), ("bf16", 1, 16, 16, 128, 63, 16), ("bf16", 1, 16, 16, 128, 64, 17),
    ("bf16", 1, 20, 4, 128, 1001, 7), ("bf16", 2, 32, 8, 128, 3001, 33), ("bf16", 1, 32, 8, 128, 9001, 130), ("bf16", 1, 17, 1, 128, 77, 3),
    ("bf16", 70, 8, 8, 128, 1000, 1), ("bf16", 70, 16, 8, 128, 65, 10), ("bf16", 40, 8, 8, 128, 700, 60),
    ("bf16", 1, 32, 8, 128, 20000, 8), ("bf16", 1, 32, 8, 128, 20000, 16), ("bf16", 1, 40, 1, 128, 40000, 1), ("bf16", 1, 8, 8, 128, 5, 300),
    # fp32
    ("fp32", 1, 1, 1, 64, 1, 1), ("fp32", 1, 1, 1, 64, 1024, 32), ("fp32", 2, 4, 2, 64, 203, 3), ("fp32", 1, 8, 2, 128, 5001, 37),
    ("fp32", 1, 8, 2, 128, 33, 1), ("fp32", 1, 5, 1, 128, 2100, 2), ("fp32", 1, 32, 8, 64, 20001, 1), ("fp32", 3, 6, 6, 128, 700, 50),
    ("fp32", 70, 8, 8, 64, 500, 1), ("fp32", 40, 8, 8, 128, 300, 40),
]


@pytest.mark.parametrize("dtype,B,Hq,Hkv,d,L,q", CALLS)
def test_append_and_attend(dtype, B, Hq, Hkv, d, L, q):
    c = Call(dtype, B, Hq, Hkv, d, L, q)
    print(f"{dtype} {B} {Hq}/{Hkv} d={d} L={L} q={q}", flush=True)
    want = c.appended()
    sa.phase2_q4(c.shape, L, c.Q, c.K, c.V, c.cache, c.O, c.ws)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(c.tensors(), want))
    c.check_O(want)


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("dtype,B,Hq,Hkv,d,L,q", CALLS[::3])
def test_one_hosts_pair(dtype, B, Hq, Hkv, d, L, q, append):
    c = Call(dtype, B, Hq, Hkv, d, L, q, seed=1)
    print(f"{dtype} {B} {Hq}/{Hkv} d={d} L={L} q={q} append={append}", flush=True)
    A, LSE = torch.full((B, Hq, q, d), math.nan).cuda(), torch.full((B, Hq, q), math.nan).cuda()
    want = c.appended() if append else [t.clone() for t in c.tensors()]
    sa.phase2_q4_partial(c.shape, L, c.Q, c.cache, A, LSE, c.ws, **(dict(Kq=c.K, Vq=c.V) if append else {}))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(c.tensors(), want))
    c.check_pair(want, A, LSE, append)


@pytest.mark.parametrize("dtype,Hq,Hkv,d,L,block,q,more", [
    ("bf16", 8, 2, 128, 1000, 256, 1, 0), ("bf16", 32, 8, 128, 5000, 700, 3, 9), ("bf16", 8, 2, 128, 300, 7, 20, 0), ("bf16", 32, 8, 128, 40000, 16384, 70, 130),
    ("fp32", 4, 1, 64, 1024, 256, 32, 5), ("fp32", 8, 2, 128, 2050, 1000, 2, 0), ("bf16", 4, 4, 128, 5, 1, 1, 0)])
def test_parts(dtype, Hq, Hkv, d, L, block, q, more):
    """Per-part pairs and their merge; `more` rows of earlier calls in the tail."""
    c = Call(dtype, 1, Hq, Hkv, d, L, q, seed=2, block=block, cached=L + more)
    n = -(-L // block)
    Op, Lp = torch.full((1, n + 1, Hq, q, d), math.nan).cuda(), torch.full((1, n + 1, Hq, q), math.nan).cuda()
    print(f"{dtype} {Hq}/{Hkv} L={L} b={block} q={q}", flush=True)
    want = c.appended()
    sa.phase2_q4(c.shape, L + more, c.Q, c.K, c.V, c.cache, c.O, c.ws, O_part=Op, LSE_part=Lp)
    torch.cuda.synchronize()
    c.check_O(want)
    for m in {0, n // 2, n - 1, n}:
        lo, hi = (m * block, min((m + 1) * block, L)) if m < n else (L, L + more + q)
        c.check_pair(want, Op[:, m], Lp[:, m], True, lo=lo, hi=hi)


@pytest.mark.parametrize("dtype,B,Hq,Hkv,d,L,q,splits,tile", [
    ("bf16", 66, 8, 8, 128, 2300, 1, 3, 16), ("bf16", 66, 16, 8, 128, 4400, 13, 3, 32), ("fp32", 65, 8, 8, 64, 2200, 2, 3, 16),
    ("bf16", 10, 32, 8, 128, 6000, 128, 3, 256), ("fp32", 40, 16, 4, 64, 3000, 30, 3, 128), ("bf16", 64, 8, 8, 128, 2000, 1, 1, 16),
    # few keys: one split, stored as it is, and the next number of them
    ("bf16", 2, 32, 8, 128, 639, 1, 1, 16), ("bf16", 1, 32, 8, 128, 640, 1, 6, 16), ("bf16", 1, 32, 8, 128, 633, 7, 1, 32), ("fp32", 1, 8, 2, 64, 300, 4, 1, 16),
    ("bf16", 1, 32, 8, 128, 200, 56, 1, 128), ("bf16", 1, 8, 8, 128, 57, 200, 3, 128), ("fp32", 1, 8, 2, 128, 190, 66, 1, 64)])
def test_more_splits_than_a_round_takes(dtype, B, Hq, Hkv, d, L, q, splits, tile):
    """More workgroups than one round, or most of one: rounds evened out by splits."""
    c = Call(dtype, B, Hq, Hkv, d, L, q, seed=16)
    p = sa.phase2_q4_plan(c.shape, L, q)
    print(f"{dtype} {B} {Hq}/{Hkv} d={d} L={L} q={q}: {p.n_splits} of {p.tile_rows}", flush=True)
    want = c.appended()
    sa.phase2_q4(c.shape, L, c.Q, c.K, c.V, c.cache, c.O, c.ws)
    A, LSE = torch.full((B, Hq, q, d), math.nan).cuda(), torch.full((B, Hq, q), math.nan).cuda()
    sa.phase2_q4_partial(c.shape, L + q, c.Q, c.cache, A, LSE, c.ws)
    torch.cuda.synchronize()
    assert (p.n_splits, p.tile_rows) == (splits, tile)
    assert all(torch.equal(x, y) for x, y in zip(c.tensors(), want))
    c.check_O(want)
    c.cached = L + q
    c.check_pair(want, A, LSE, False)


def test_pairs_of_two_hosts_merge_to_the_whole():
    whole = Call("bf16", 1, 8, 2, 128, 900, 5, seed=3)
    tensors, pairs = whole.appended(), []
    for lo, hi in ((0, 400), (400, 900)):
        last = hi == 900
        shape = sa.StarShape.make("bf16", 1, 8, 2, 128, hi - lo, hi - lo, 0, hi - lo + 5)
        cache = sa.alloc_q4_cache(shape)
        for to, x in zip((cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), whole.tensors()):
            to[:, :, :hi - lo] = x[:, :, lo:hi]
        A, LSE = torch.empty(1, 8, 5, 128).cuda(), torch.empty(1, 8, 5).cuda()
        sa.phase2_q4_partial(shape, hi - lo, whole.Q, cache, A, LSE, sa.alloc_q4_workspace(shape, 5), **(dict(Kq=whole.K, Vq=whole.V) if last else {}))
        pairs.append((A, LSE))
    A, LSE = (torch.stack(x).contiguous() for x in zip(*pairs))
    sa.merge(whole.shape, A, LSE, O=whole.O)
    torch.cuda.synchronize()
    whole.check_O(tensors, few=8)


@pytest.mark.parametrize("dtype,Hq,Hkv,d,L,q", [("bf16", 8, 2, 128, 300, 3), ("bf16", 8, 2, 128, 300, 30), ("fp32", 4, 2, 64, 203, 40), ("bf16", 8, 2, 128, 3000, 90)])
def test_not_finite_values_count_for_the_rows_that_see_them(dtype, Hq, Hkv, d, L, q):
    """An infinity in a new token's V, a NaN in another's K: earlier tokens of the call do not see them."""
    c = Call(dtype, 1, Hq, Hkv, d, L, q, seed=4)
    c.V[:, q - 1, 0, 5] = math.inf
    c.K[:, q - 1, 1, d - 1] = math.nan
    c.V[:, q // 2, 1, d - 3] = math.nan
    want = c.appended()
    print(f"{dtype} {Hq}/{Hkv} L={L} q={q}", flush=True)
    sa.phase2_q4(c.shape, L, c.Q, c.K, c.V, c.cache, c.O, c.ws)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(c.tensors(), want))
    O = c.O[0]
    assert torch.isfinite(O[:q // 2].float()).all()
    assert O[q - 1, 0, :32].isnan().all() and torch.isfinite(O[q - 1, 0, 32:].float()).all()
    assert O[q - 1, Hq - 1].isnan().all()                        # a logit that is NaN
    assert O[q // 2, Hq - 1, d - 32:].isnan().all() and torch.isfinite(O[q // 2, Hq - 1, :d - 32].float()).all()
    if q // 2 < q - 1:
        assert torch.isfinite(O[q - 2, 0].float()).all()


def test_values_and_queries_far_from_one():
    """Units next to both ends of their range, logits of hundreds."""
    c = Call("bf16", 1, 8, 2, 128, 400, 2, seed=5)
    c.V[:, 0] = 3e38
    c.V[:, 1] *= 1e-37
    c.Q *= 60
    want = c.appended()
    sa.phase2_q4(c.shape, 400, c.Q, c.K, c.V, c.cache, c.O, c.ws)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(c.tensors(), want))
    c.check_O(want, few=8)


@pytest.mark.parametrize("at", ["first", "middle", "last", "new"])
@pytest.mark.parametrize("dtype,Hq,Hkv,d,L,q", [("bf16", 8, 2, 128, 900, 3), ("bf16", 8, 2, 128, 900, 7), ("bf16", 8, 2, 128, 2000, 70),
                                                ("bf16", 32, 8, 128, 3000, 128), ("fp32", 4, 2, 64, 900, 4), ("fp32", 8, 2, 128, 900, 40)])
def test_values_that_fp16_does_not_hold(dtype, Hq, Hkv, d, L, q, at):
    """Units of V past 2^13 and below 2^-23, in cached rows and in the call's own; a key whose group is NaN among the cached."""
    c = Call(dtype, 1, Hq, Hkv, d, L, q, seed=10)
    print(f"{dtype} {Hq}/{Hkv} L={L} q={q} {at}", flush=True)
    if at == "new":
        c.V[:, 0, 0] *= 2.0 ** 20
        c.V[:, q - 1, 1] *= 2.0 ** -60
    else:
        row = {"first": 0, "middle": L // 2, "last": L - 1}[at]
        c.cache.v_scales[0, 0, row] += 30
        c.cache.v_scales[0, 1, row, 1] -= 50
    want = c.appended()
    sa.phase2_q4(c.shape, L, c.Q, c.K, c.V, c.cache, c.O, c.ws)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(c.tensors(), want))
    c.check_O(want, few=8)
    A, LSE = torch.empty((1, Hq, q, d)).cuda(), torch.empty((1, Hq, q)).cuda()
    sa.phase2_q4_partial(c.shape, L, c.Q, c.cache, A, LSE, c.ws, Kq=c.K, Vq=c.V)
    torch.cuda.synchronize()
    c.check_pair(want, A, LSE, True, few=8)
    if at != "new":
        c.cache.v_scales[0, 0, row, 0], c.cache.k_scales[0, 1, row, 0] = 255, 255
        sa.phase2_q4(c.shape, L, c.Q, c.K, c.V, c.cache, c.O, c.ws)
        torch.cuda.synchronize()
        G = Hq // Hkv
        nan = c.O[0].isnan()
        assert nan[:, :G, :32].all() and not nan[:, :G, 32:].any() and nan[:, G:2 * G].all() and not nan[:, 2 * G:].any()


@pytest.mark.parametrize("dtype,Hq,Hkv,d,L,q", [("bf16", 8, 2, 128, 900, 3), ("bf16", 8, 2, 128, 6000, 70), ("fp32", 8, 2, 128, 900, 40)])
def test_scores_that_rise_all_along(dtype, Hq, Hkv, d, L, q):
    """Each key's logit above the one before, by 2^9 in all: the references move, everywhere, and what was summed up before fades."""
    c = Call(dtype, 1, Hq, Hkv, d, L, q, seed=11)
    c.Q.fill_(1.0)
    K = (torch.arange(L)[:, None] / L * 45 * torch.ones(d))[None, None].expand(1, Hkv, L, d)
    codes, scales = star_q4.quantise(K)
    c.cache.k_codes[:, :, :L], c.cache.k_scales[:, :, :L] = codes.cuda(), scales.cuda()
    want = c.appended()
    sa.phase2_q4(c.shape, L, c.Q, c.K, c.V, c.cache, c.O, c.ws)
    torch.cuda.synchronize()
    c.check_O(want, few=8)


def test_captured_and_replayed():
    """Every replay, with eager work in between, gives the eager call's bits; two graphs with workspaces of their own."""
    one, two = Call("bf16", 1, 32, 8, 128, 3000, 1, seed=6), Call("bf16", 1, 8, 2, 128, 700, 20, seed=7)
    eager = []
    for c in (one, two):
        c.start = [t.clone() for t in c.tensors()]
        sa.phase2_q4(c.shape, c.cached, c.Q, c.K, c.V, c.cache, c.O, c.ws)
        eager.append((c.O.clone(), [t.clone() for t in c.tensors()]))
    torch.cuda.synchronize()
    graphs = []
    for c in (one, two):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sa.phase2_q4(c.shape, c.cached, c.Q, c.K, c.V, c.cache, c.O, c.ws)
        graphs.append(g)
    for _ in range(4):
        for c in (one, two):
            c.O.fill_(math.nan)
            for t, s in zip(c.tensors(), c.start):
                t.copy_(s)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for c, (O, tensors) in zip((one, two), eager):
            assert torch.equal(c.O, O) and all(torch.equal(x, y) for x, y in zip(c.tensors(), tensors))


def test_calls_on_two_streams():
    calls = [Call("bf16", 1, 32, 8, 128, 6000 + 500 * i, 1 + 30 * i, seed=8) for i in range(2)]
    for c in calls:
        sa.phase2_q4(c.shape, c.cached, c.Q, c.K, c.V, c.cache, c.O, c.ws)
    torch.cuda.synchronize()
    want = [c.O.clone() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        for c in calls:
            c.O.fill_(math.nan)
        torch.cuda.synchronize()
        for c, s in zip(calls, streams):
            sa.phase2_q4(c.shape, c.cached, c.Q, c.K, c.V, c.cache, c.O, c.ws, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(c.O, w) for c, w in zip(calls, want))


@pytest.mark.parametrize("dtype,B,Hq,Hkv,d,L,q", [("bf16", 1, 8, 2, 128, 900, 6), ("bf16", 70, 8, 8, 128, 90, 2), ("bf16", 3, 8, 8, 128, 100, 100),
                                                  ("fp32", 70, 8, 8, 64, 200, 3)])
@pytest.mark.parametrize("over", ["Q", "K", "V"])
def test_output_over_what_is_read(dtype, B, Hq, Hkv, d, L, q, over):
    """With many splits, and with one, whose workgroups store the output themselves."""
    c = Call(dtype, B, Hq, Hkv, d, L, q, seed=9)
    if over != "Q" and Hq != Hkv:
        pytest.skip("sizes differ")
    want = c.appended()
    print(f"{dtype} {B} {Hq}/{Hkv} L={L} q={q} over {over}", flush=True)
    Q, K, V = c.Q.clone(), c.K.clone(), c.V.clone()
    O = {"Q": Q, "K": K, "V": V}[over]
    sa.phase2_q4(c.shape, L, Q, K, V, c.cache, O, c.ws)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(c.tensors(), want))
    c.O = O
    c.check_O(want)


@pytest.mark.parametrize("L,q", [(100, 1), (60, 40), (3000, 2)])
@pytest.mark.parametrize("over", ["Q", "K"])
def test_pair_over_what_is_read(L, q, over):
    """In fp32 a pair's outputs fit where its queries or keys were."""
    c = Call("fp32", 2, 4, 4, 64, L, q, seed=17)
    want = c.appended()
    print(f"L={L} q={q} over {over}", flush=True)
    X = {"Q": c.Q, "K": c.K}[over].clone()
    A, LSE = X.view(2, 4, q, 64), torch.full((2, 4, q), math.nan).cuda()
    sa.phase2_q4_partial(c.shape, L, X if over == "Q" else c.Q, c.cache, A, LSE, c.ws, Kq=X if over == "K" else c.K, Vq=c.V)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(c.tensors(), want))
    c.check_pair(want, A, LSE, True, few=8)


def _rows_of(c, q, tensors, b, h, j):
    """Token j's row of a long call against the oracle, in units of its bound."""
    B, Hq, Hkv, d = c.dims
    g, n = h // (Hq // Hkv), c.cached + j + 1
    K, V = (star_q4.values(tensors[i][b, g, :n], tensors[i + 1][b, g, :n]) for i in (0, 2))
    A, lse, weights, size, total = star_q4.attend(c.Q[b, j:j + 1, h], K, V, c.scale)
    bound = _bound("bf16", d, n, size, weights, total, 1) + A.abs() * 2.0 ** -8
    return ((c.O[b, j:j + 1, h].double() - A).abs() / bound).max().item()


@pytest.mark.parametrize("q", [1, 4200])
def test_bytes_past_32_bits(q):
    """64 sequences whose codes lie past 2^32 bytes, one token each and calls whose queries do as well."""
    B, Hq, Hkv, d, L, cap = 64, 64, 8, 128, 70, 140000
    gen = torch.Generator(device="cuda").manual_seed(2)
    rand = lambda *size: torch.randn(*size, generator=gen, device="cuda", dtype=torch.bfloat16)
    c = Call.__new__(Call)
    c.cached, c.q, c.dims, c.dtype, c.scale = L, q, (B, Hq, Hkv, d), "bf16", d ** -0.5
    c.shape = sa.StarShape.make("bf16", B, Hq, Hkv, d, L, L, 0, cap)
    c.Q, c.K, c.V, c.cache = rand(B, q, Hq, d), rand(B, q, Hkv, d), rand(B, q, Hkv, d), sa.alloc_q4_cache(c.shape)
    assert c.cache.k_codes.numel() > 2 ** 32 and (q == 1 or c.Q.numel() > 2 ** 31)
    Kc, Vc = rand(B, Hkv, L, d), rand(B, Hkv, L, d)
    sa.q4_store(c.shape, 0, L, Kc, Vc, c.cache)
    c.O = torch.full_like(c.Q, math.nan)
    ws = torch.empty(sa.phase2_q4_plan(c.shape, L, q).workspace_bytes, dtype=torch.uint8, device="cuda")
    sa.phase2_q4(c.shape, L, c.Q, c.K, c.V, c.cache, c.O, ws)
    Kb, Vb = torch.empty_like(Kc), torch.empty_like(Vc)
    sa.q4_load(c.shape, 0, L, c.cache, Kb, Vb)
    torch.cuda.synchronize()
    tensors = c.tensors()
    for b in (0, 31, B - 1):
        for plain, back, new, i in ((Kc, Kb, c.K, 0), (Vc, Vb, c.V, 2)):
            codes, scales = star_q4.quantise(torch.cat([plain[b], new[b].transpose(0, 1)], 1))
            assert torch.equal(tensors[i][b, :, :L + q], codes) and torch.equal(tensors[i + 1][b, :, :L + q], scales)
            assert torch.equal(back[b].double(), star_q4.values(codes[:, :L], scales[:, :L]))
            assert (tensors[i][b, :, L + q:L + q + 99] == 0).all()
        for h, j in ((0, 0), (Hq - 1, q - 1), (9, q // 2)):
            assert _rows_of(c, q, tensors, b, h, j) <= 1, (b, h, j)


@pytest.mark.parametrize("q", [1, 20, 40, 300])
def test_a_cache_of_one_head_past_32_bits(q):
    """70 million keys, zeros but for some at the end and at both sides of byte 2^31 and 2^32 of the codes."""
    d, L = 128, 70000000
    shape = sa.StarShape.make("bf16", 1, 1, 1, d, L, L, 0, L + q)
    cache = sa.alloc_q4_cache(shape)
    assert cache.k_codes.numel() > 2 ** 32
    cache.k_scales.fill_(127), cache.v_scales.fill_(127)
    gen = torch.Generator().manual_seed(q)
    Q, K, V = (_randn(gen, "bf16", 1, q, 1, d) for _ in range(3))
    Q = Q * 4
    spots, n = [2 ** 31 // 64 - 40, 2 ** 32 // 64 - 40, L - 80], 80
    plain = [_randn(gen, "bf16", 1, 1, n, d) for _ in range(6)]
    for i, at in enumerate(spots):
        sa.q4_store(shape, at, n, plain[2 * i], plain[2 * i + 1], cache, plain_row=0)
    O = torch.full_like(Q, math.nan)
    sa.phase2_q4(shape, L, Q, K, V, cache, O, sa.alloc_q4_workspace(shape, q))
    A, LSE = torch.empty(1, 1, q, d).cuda(), torch.empty(1, 1, q).cuda()
    sa.phase2_q4_partial(shape, L, Q, cache, A, LSE, sa.alloc_q4_workspace(shape, q))
    torch.cuda.synchronize()
    k, v = (star_q4.values(*star_q4.quantise(torch.cat([*(x[0, 0] for x in plain[i::2]), X[0, :, 0]]))) for i, X in ((0, K), (1, V)))
    assert torch.equal(star_q4.values(cache.v_codes[0, 0, L:], cache.v_scales[0, 0, L:]), v[3 * n:])
    zeros = L - 3 * n
    for j in (0, q // 2, q - 1):
        x = Q[0, j, 0].double()
        for last, got, half in ((3 * n + j + 1, O[0, j, 0], 2.0 ** -8), (3 * n, A[0, 0, j], 2.0 ** -16)):
            s = k[:last] @ x * d ** -0.5
            size = (k[:last].abs() @ x.abs()).max() * d ** -0.5
            lse = torch.logsumexp(torch.cat([s, torch.tensor([math.log(zeros)], dtype=torch.float64).cuda()]), 0)
            p = torch.exp(s - lse)
            want, weights, total = p @ v[:last], p @ v[:last].abs(), v[:last].abs().sum(0)
            bound = _bound("bf16", d, L, size[None], weights[None], total[None], 1 if half > 1e-3 else 2)[0] + want.abs() * (half if half > 1e-3 else 2.0 ** -24)
            assert ((got.double() - want).abs() <= bound).all(), (j, last)
        assert abs(LSE[0, 0, j].double() - lse) <= 2.0 ** -24 * (2 * (d + 4) * size + L / 32 + 64 + 8 * lse.abs())
