"""Queries and keys normed per head and rotated on one or several axes, against 64 bits (oracle/star_q4.py), and the calls
that do it on the way against the same in steps.

Bounds: a row's mean square is d products summed in 32 bits (d 2^-24 at most, halved by the root), division, root, the two factors and
the weight round once each, cosine and sine once, their products and the sum twice: (d / 2 + 10) 2^-24 of |n_i| + |n_(i + d/2)|.
Then half a step of the storage type, 2^-8 or 2^-24 of the result."""
import math

import pytest
import torch

import paper_2411_17116_amd as sa
from oracle import star_q4

pytestmark = pytest.mark.gpu

THETA = 500000.0


def _dt(dtype):
    return torch.float32 if dtype == "fp32" else torch.bfloat16


def _randn(gen, dtype, *size):
    return torch.randn(size, generator=gen).to(_dt(dtype)).cuda()


def _near(got, x, weight, eps, positions, axis, dtype, theta=THETA):
    want, pair = star_q4.norm_rope(x, weight, eps, theta, positions, axis)
    d = x.shape[-1]
    bound = torch.cat([pair, pair], -1) * (d / 2 + 10) * 2.0 ** -24 + want.abs() * (2.0 ** -24 if dtype == "fp32" else 2.0 ** -8) + 1e-37
    off = (got.double() - want).abs()
    assert (off <= bound).all(), ((off / bound).max().item(), off.max().item())


# tokens on either side of where a workgroup takes 1, 4 or 16 of them, odd heads
@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,d", [
    ("bf16", 1, 1, 32, 8, 128), ("bf16", 1, 1, 1, 1, 128), ("bf16", 3, 7, 5, 1, 128), ("bf16", 2, 1025, 4, 2, 128), ("bf16", 1, 4099, 2, 1, 128),
    ("bf16", 1, 1500, 32, 8, 128), ("fp32", 1, 1, 8, 2, 64), ("fp32", 2, 33, 3, 3, 64), ("fp32", 1, 1030, 4, 1, 128), ("fp32", 2, 2100, 1, 1, 64)])
@pytest.mark.parametrize("axes", [1, 3])
def test_pass(dtype, B, T, Hq, Hkv, d, axes):
    gen = torch.Generator().manual_seed(T + Hq)
    size = torch.exp(torch.randn(B, T, 1, 1, generator=gen) * 2).cuda()
    Q, K = ((_randn(gen, dtype, B, T, H, d) * size).to(_dt(dtype)) for H in (Hq, Hkv))
    wq, wk = (1 + torch.randn(d, generator=gen) / 4).to(_dt(dtype)).cuda(), (1 + torch.randn(d, generator=gen) / 4).to(_dt(dtype)).cuda()
    shape = sa.StarShape.make(dtype, B, Hq, Hkv, d, 5, 5, 0, 5)
    if axes == 1:
        rotary = sa.Rotary(THETA, q_norm=wq, k_norm=wk, eps=1e-5, pos0=1000003)
        positions, axis = torch.arange(T).expand(B, T)[..., None] + 1000003, [0] * (d // 2)
    else:
        positions = torch.randint(-50, 200000, (B, T, 3), generator=gen)
        sections = [d // 8, d // 4 - 3, d // 8 + 3]
        axis = [a for a, n in enumerate(sections) for _ in range(n)]
        rotary = sa.Rotary(THETA, q_norm=wq, k_norm=wk, eps=1e-5, positions=positions.cuda(), sections=sections)
    print(f"{dtype} {B} {T} {Hq}/{Hkv} {d} axes={axes}", flush=True)
    Yq, Yk = torch.full_like(Q, math.nan), torch.full_like(K, math.nan)
    sa.qk_norm_rope(shape, rotary, Q, K, Yq, Yk)
    torch.cuda.synchronize()
    _near(Yq, Q, wq, 1e-5, positions.cuda(), axis, dtype)
    _near(Yk, K, wk, 1e-5, positions.cuda(), axis, dtype)
    # one of them alone, in place, on a stream of its own: the same bits
    stream = torch.cuda.Stream()
    X, Z = Q.clone(), K.clone()
    torch.cuda.synchronize()
    sa.qk_norm_rope(shape, rotary, X, None, X, None, stream=stream)
    sa.qk_norm_rope(shape, rotary, None, Z, None, Z, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(X, Yq) and torch.equal(Z, Yk)


def test_positions_of_any_token_of_a_longer_tensor():
    """A decode step's positions cut out of a prompt's: whole numbers, not 16 bytes, apart."""
    gen = torch.Generator().manual_seed(22)
    every = torch.randint(0, 4000, (1, 20, 3), generator=gen).cuda()
    Q = _randn(gen, "bf16", 1, 2, 4, 128)
    shape = sa.StarShape.make("bf16", 1, 4, 2, 128, 5, 5, 0, 5)
    axis = [i % 3 for i in range(64)]
    for t in (1, 2, 7, 18):
        Y = torch.empty_like(Q)
        sa.qk_norm_rope(shape, sa.Rotary(THETA, positions=every[:, t:t + 2], axis=axis), Q, None, Y, None)
        torch.cuda.synchronize()
        _near(Y, Q, None, 0.0, every[:, t:t + 2], axis, "bf16")


def test_axes_dealt_in_turn_and_four_of_them():
    gen = torch.Generator().manual_seed(1)
    Q, K = _randn(gen, "bf16", 2, 9, 4, 128), _randn(gen, "bf16", 2, 9, 2, 128)
    shape = sa.StarShape.make("bf16", 2, 4, 2, 128, 5, 5, 0, 5)
    for n in (2, 4):
        positions = torch.randint(0, 1 << 20, (2, 9, n), generator=gen).cuda()
        axis = [(3 * i + i // 7) % n for i in range(64)]
        Yq, Yk = torch.empty_like(Q), torch.empty_like(K)
        sa.qk_norm_rope(shape, sa.Rotary(10000.0, positions=positions, axis=axis), Q, K, Yq, Yk)
        torch.cuda.synchronize()
        _near(Yq, Q, None, 0.0, positions, axis, "bf16", 10000.0)
        _near(Yk, K, None, 0.0, positions, axis, "bf16", 10000.0)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64), ("fp32", 128)])
def test_without_norms_on_one_axis_the_rotation_alone(dtype, d):
    gen = torch.Generator().manual_seed(2)
    Q, K = _randn(gen, dtype, 1, 77, 8, d), _randn(gen, dtype, 1, 77, 2, d)
    shape = sa.StarShape.make(dtype, 1, 8, 2, d, 5, 5, 0, 5)
    Yq, Yk, Rq, Rk = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(Q), torch.empty_like(K)
    sa.rope(shape, Q, Rq, THETA, pos0=41)
    sa.rope(shape, K, Rk, THETA, pos0=41)
    sa.qk_norm_rope(shape, sa.Rotary(THETA, pos0=41), Q, K, Yq, Yk)
    positions = torch.arange(41, 118)[None].cuda()
    Zq, Zk = torch.empty_like(Q), torch.empty_like(K)
    sa.qk_norm_rope(shape, sa.Rotary(THETA, positions=positions), Q, K, Zq, Zk)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in ((Yq, Rq), (Yk, Rk), (Zq, Rq), (Zk, Rk)))


def test_rows_of_zeros_large_and_small_ones_and_nan():
    gen = torch.Generator().manual_seed(3)
    Q = _randn(gen, "fp32", 1, 6, 3, 64)
    Q[0, 0], Q[0, 1, 1], Q[0, 2, 0], Q[0, 3, 2, 5] = 0.0, Q[0, 1, 1] * 1e15, Q[0, 2, 0] * 1e-15, math.nan
    w = torch.ones(64).cuda()
    shape = sa.StarShape.make("fp32", 1, 3, 3, 64, 5, 5, 0, 5)
    Y = torch.empty_like(Q)
    sa.qk_norm_rope(shape, sa.Rotary(THETA, q_norm=w, eps=1e-6), Q, None, Y, None)
    torch.cuda.synchronize()
    assert (Y[0, 0] == 0).all() and Y[0, 3, 2].isnan().all() and Y.isnan().sum() == 64
    Q[0, 3, 2, 5] = 0.0
    sa.qk_norm_rope(shape, sa.Rotary(THETA, q_norm=w, eps=1e-6), Q, None, Y, None)
    torch.cuda.synchronize()
    _near(Y, Q, w, 1e-6, torch.arange(6)[None, :, None].cuda(), [0] * 32, "fp32")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64), ("fp32", 128)])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_rows_whose_squares_32_bits_do_not_hold(dtype, d, eps):
    """Sizes from the storage type's largest to its least normal ones, in one workgroup; an infinity takes its row to zeros and,
    where its pair is rotated to, NaN."""
    gen = torch.Generator().manual_seed(21)
    sizes = torch.tensor([2.0 ** e for e in (124, 80, 64, 58, 0, -45, -52, -60, -80, -110, -124)])
    X = torch.rand(1, 3, len(sizes), d, generator=gen) + 0.5
    X = (X * torch.sign(torch.randn(X.shape, generator=gen)) * sizes[:, None]).to(_dt(dtype)).cuda()
    w = (1 + torch.randn(d, generator=gen) / 4).to(_dt(dtype)).cuda()
    shape = sa.StarShape.make(dtype, 1, len(sizes), 1, d, 5, 5, 0, 5)
    Y = torch.full_like(X, math.nan)
    rotary = sa.Rotary(THETA, q_norm=w, eps=eps, pos0=3)
    sa.qk_norm_rope(shape, rotary, X, None, Y, None)
    torch.cuda.synchronize()
    _near(Y, X, w, eps, torch.arange(3, 6)[None, :, None].cuda(), [0] * (d // 2), dtype)
    X[0, 1, 4, 7] = math.inf
    sa.qk_norm_rope(shape, rotary, X, None, Y, None)
    torch.cuda.synchronize()
    bad = Y.isnan()
    assert bad.sum() == 2 and bad[0, 1, 4, 7] and bad[0, 1, 4, 7 + d // 2]
    assert (Y[0, 1, 4][~bad[0, 1, 4]] == 0).all()


def test_captured_and_replayed():
    """The pass, both phases on projections and rows filed and read, captured together: replays among eager work give the
    eager call's bits."""
    L, q, Hq, Hkv, d = 900, 5, 8, 2, 128
    Q, K, V, kw = _setup("bf16", 2, Hq, Hkv, d, L + q, 14, True)
    shape = sa.StarShape.make("bf16", 2, Hq, Hkv, d, L, 300, 100, L + q)
    cut = lambda X, lo, hi: X[:, lo:hi].clone()
    positions = kw.pop("positions")
    context, question = (sa.Rotary(THETA, positions=positions[:, s].contiguous(), **kw) for s in (slice(0, L), slice(L, None)))
    first, then = [cut(X, 0, L) for X in (Q, K, V)], [cut(X, L, L + q) for X in (Q, K, V)]
    work = [torch.empty_like(first[0]), torch.empty_like(then[0]), torch.empty_like(then[0])]
    Kc, Vc = sa.alloc_cache(shape)
    Kb, Vb = sa.alloc_cache(shape)
    cache, O, Oq, O4 = sa.alloc_q4_cache(shape), torch.empty_like(first[0]), torch.empty_like(then[0]), torch.empty_like(then[0])
    Yk, ws, ws2 = torch.empty_like(first[1]), sa.alloc_workspace(shape, q), sa.alloc_q4_workspace(shape, q)
    out = [*work, Kc, Vc, Kb, Vb, cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales, O, Oq, O4, Yk]
    ws1 = sa.alloc_workspace(shape, L)

    def run():
        work[0].copy_(first[0]), work[1].copy_(then[0]), work[2].copy_(then[0])
        sa.qk_norm_rope(shape, context, None, first[1], None, Yk)
        sa.phase1_norm_rope(shape, context, work[0], first[1], first[2], O, Kc, Vc, workspace=ws1)
        sa.q4_store(shape, 0, L, Kc, Vc, cache)
        sa.phase2_norm_rope(shape, question, L, work[1], then[1], then[2], Kc, Vc, Oq, ws)
        sa.phase2_q4(shape, L, work[2], then[1], then[2], cache, O4, ws2, rotary=question)
        sa.q4_load(shape, 0, L + q, cache, Kb, Vb)

    for t in out:
        t.zero_()
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        for t in out:
            t.fill_(7 * i + 1)
        for t in (Kc, Vc, Kb, Vb):
            t.zero_()
        for t in out[7:11]:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want))


def test_on_two_streams_at_once():
    gen = torch.Generator().manual_seed(15)
    shape = sa.StarShape.make("bf16", 1, 32, 8, 128, 5, 5, 0, 5)
    w = torch.ones(128).bfloat16().cuda()
    calls = [(_randn(gen, "bf16", 1, T, 32, 128), _randn(gen, "bf16", 1, T, 8, 128), sa.Rotary(THETA, q_norm=w, k_norm=w, pos0=T)) for T in (3000, 700)]
    want, got = [], []
    for Q, K, r in calls:
        want.append((torch.empty_like(Q), torch.empty_like(K)))
        got.append((torch.empty_like(Q), torch.empty_like(K)))
        sa.qk_norm_rope(shape, r, Q, K, *want[-1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        for (Q, K, r), y, s in zip(calls, got, streams):
            y[0].zero_(), y[1].zero_()
        torch.cuda.synchronize()
        for (Q, K, r), y, s in zip(calls, got, streams):
            sa.qk_norm_rope(shape, r, Q, K, *y, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(x, z) for a, b in zip(got, want) for x, z in zip(a, b))


def _setup(dtype, B, Hq, Hkv, d, T, seed, pos=None):
    gen = torch.Generator().manual_seed(seed)
    Q, K, V = (_randn(gen, dtype, B, T, H, d) for H in (Hq, Hkv, Hkv))
    wq, wk = (1 + torch.randn(d, generator=gen) / 4).to(_dt(dtype)).cuda(), (1 + torch.randn(d, generator=gen) / 4).to(_dt(dtype)).cuda()
    positions = torch.randint(0, 5000, (B, T, 3), generator=gen).cuda() if pos else None
    kw = dict(q_norm=wq, k_norm=wk, eps=1e-6)
    if pos:
        kw.update(positions=positions, sections=[d // 8, d // 4, d // 8])
    return Q, K, V, kw


@pytest.mark.parametrize("dtype,B,Hq,Hkv,d,L,block,a,pos", [
    ("bf16", 1, 8, 2, 128, 1000, 256, 100, False), ("bf16", 2, 8, 2, 128, 700, 300, 300, True), ("fp32", 1, 4, 2, 64, 500, 128, 128, True)])
def test_phase1_in_steps(dtype, B, Hq, Hkv, d, L, block, a, pos):
    Q, K, V, kw = _setup(dtype, B, Hq, Hkv, d, L, 11, pos)
    shape = sa.StarShape.make(dtype, B, Hq, Hkv, d, L, block, a, L + 9)
    rotary = sa.Rotary(THETA, pos0=0 if pos else 17, **kw)
    Yq, Yk = torch.empty_like(Q), torch.empty_like(K)
    sa.qk_norm_rope(shape, rotary, Q, K, Yq, Yk)
    outs = []
    for i in range(2):
        Kc, Vc = sa.alloc_cache(shape)
        Kc.fill_(3.0), Vc.fill_(3.0)
        O, LSE = torch.empty_like(Q), torch.empty(B, Hq, L).cuda()
        X = Q.clone()
        if i == 0:
            sa.phase1(shape, Yq, Yk, V, O, Kc, Vc, LSE_ctx=LSE)
        else:
            sa.phase1_norm_rope(shape, rotary, X, K, V, O, Kc, Vc, LSE_ctx=LSE)
        outs.append((O, LSE, Kc, Vc))
    torch.cuda.synchronize()
    assert torch.equal(X, Yq)
    assert all(torch.equal(x, y) for x, y in zip(*outs))


@pytest.mark.parametrize("dtype,B,Hq,Hkv,d,L,q,pos", [
    ("bf16", 1, 8, 2, 128, 1000, 1, False), ("bf16", 2, 8, 2, 128, 3000, 5, True), ("bf16", 1, 32, 8, 128, 2000, 40, True), ("fp32", 1, 4, 2, 64, 500, 3, False)])
@pytest.mark.parametrize("q4", [False, True])
def test_phase2_in_steps(dtype, B, Hq, Hkv, d, L, q, pos, q4):
    """Over a plain and a four-bit cache."""
    Q, K, V, kw = _setup(dtype, B, Hq, Hkv, d, q, 12, pos)
    shape = sa.StarShape.make(dtype, B, Hq, Hkv, d, L, L, 0, L + q + 3)
    gen = torch.Generator().manual_seed(5)
    Kc, Vc = (_randn(gen, dtype, B, Hkv, L + q + 3, d) for _ in range(2))
    rotary = sa.Rotary(THETA, pos0=5, **kw)
    step = rotary if pos else sa.Rotary(THETA, pos0=5 + L, **kw)
    Yq, Yk = torch.empty_like(Q), torch.empty_like(K)
    sa.qk_norm_rope(shape, step, Q, K, Yq, Yk)
    outs, X = [], Q.clone()
    print(f"{dtype} {B} {Hq}/{Hkv} {L} {q} q4={q4}", flush=True)
    for i in range(2):
        O = torch.empty_like(Q)
        if q4:
            cache = sa.alloc_q4_cache(shape)
            sa.q4_store(shape, 0, L + q + 3, Kc, Vc, cache)
            ws = sa.alloc_q4_workspace(shape, q)
            if i == 0:
                sa.phase2_q4(shape, L, Yq, Yk, V, cache, O, ws)
            else:
                sa.phase2_q4(shape, L, X, K, V, cache, O, ws, rotary=rotary)
            outs.append((O, cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales))
        else:
            kc, vc, ws = Kc.clone(), Vc.clone(), sa.alloc_workspace(shape, q)
            if i == 0:
                sa.phase2(shape, L, Yq, Yk, V, kc, vc, O, ws)
            else:
                sa.phase2_norm_rope(shape, rotary, L, X, K, V, kc, vc, O, ws)
            outs.append((O, kc, vc))
    torch.cuda.synchronize()
    assert torch.equal(X, Yq)
    assert all(torch.equal(x, y) for x, y in zip(*outs))


def test_elements_past_32_bits():
    """Projections of 2^32 bytes and more: the last tokens, and those about 2^31 elements."""
    T, Hq, d = 270000, 64, 128
    shape = sa.StarShape.make("bf16", 1, Hq, 1, d, 5, 5, 0, 5)
    gen = torch.Generator(device="cuda").manual_seed(1)
    Q = torch.randn(1, T, Hq, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(d).bfloat16().cuda()
    Y = torch.empty_like(Q)
    sa.qk_norm_rope(shape, sa.Rotary(THETA, q_norm=w), Q, None, Y, None)
    torch.cuda.synchronize()
    edge = 2 ** 31 // (Hq * d)
    for t in (0, edge - 3, T - 6):
        _near(Y[:, t:t + 6], Q[:, t:t + 6], w, 1e-6, torch.arange(t, t + 6)[None, :, None].cuda(), [0] * 64, "bf16")


def test_a_serving_run():
    """Phase 1 on projections, its cache put into four bits, a question and decode steps: every output against 64 bits over
    what the cache holds, and the rows of the cache against the steps' own keys."""
    L, lq, steps, Hq, Hkv, d = 1500, 20, 4, 8, 2, 128
    Q, K, V, kw = _setup("bf16", 1, Hq, Hkv, d, L + lq + steps, 13)
    shape = sa.StarShape.make("bf16", 1, Hq, Hkv, d, L, 400, 200, L + lq + steps)
    rotary = sa.Rotary(THETA, **kw)
    part = lambda X, lo, hi: X[:, lo:hi].clone()
    Kc, Vc = sa.alloc_cache(shape)
    O = torch.empty_like(Q[:, :L])
    sa.phase1_norm_rope(shape, rotary, part(Q, 0, L), part(K, 0, L), part(V, 0, L), O, Kc, Vc)
    cache = sa.alloc_q4_cache(shape)
    sa.q4_store(shape, 0, L, Kc, Vc, cache)
    ws = sa.alloc_q4_workspace(shape, lq)
    at = L
    Yq, Yk = torch.empty_like(Q), torch.empty_like(K)
    sa.qk_norm_rope(shape, rotary, Q, K, Yq, Yk)
    for n in [lq] + [1] * steps:
        q = part(Q, at, at + n)
        out = torch.empty_like(q)
        sa.phase2_q4(shape, at, q, part(K, at, at + n), part(V, at, at + n), cache, out, ws, rotary=rotary)
        torch.cuda.synchronize()
        assert torch.equal(q, Yq[:, at:at + n])
        for h in (0, Hq - 1):
            g = h // (Hq // Hkv)
            k, e = star_q4.quantise(Yk[0, :at + n, g])
            assert torch.equal(cache.k_codes[0, g, :at + n], k) and torch.equal(cache.k_scales[0, g, :at + n], e)
            v, f = star_q4.quantise(V[0, :at + n, g])
            A, _, weights, size, total = star_q4.attend(q[0, :, h], star_q4.values(k, e), star_q4.values(v, f), d ** -0.5, at)
            bound = weights * (2.0 ** -8 + 2.0 ** -23 * ((d + 4) * size[:, None] + at / 32 + 64)) + total * 2.0 ** -35 + A.abs() * 2.0 ** -8
            assert ((out[0, :, h].double() - A).abs() <= bound).all()
        at += n
