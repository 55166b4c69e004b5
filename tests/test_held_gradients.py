"""Gradients that the caller holds: norms, clip-weighted sums and scaled gradients of many tensors against their definitions in 64 bits.

Tolerances.  u = 2^-24 is the most that one fp32 operation is off, relative to its result.  A squared norm adds non-negative terms: off by u for
every addition on the longest path of an element through the sum.  That path is at most 9 additions in a thread (8,192 elements of a workgroup, 256
threads, 4 chains), 9 over the workgroup, and over the partial sums of up to 1,400 pieces at most 22 in a lane and 6 over the lanes, next to the
square itself: below 64 at these sizes.  A clip factor has half the norm's error and two roundings; a weighted sum of B terms adds at most
B / 4 + 20 roundings, each relative to the sum of the terms' magnitudes.  A result of fewer bits is rounded once, by at most half its eps."""
import ctypes

import numpy as np
import pytest
import torch

from gpu_util import DEV

U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _tensors(B, counts, dtype, seed, offset=0):
    """[B, count] tensors, `offset` elements behind the 16-byte boundary that an allocation begins at, and scales from clipped to not."""
    g = torch.Generator().manual_seed(seed)
    scale = torch.logspace(-1.5, 1.5, B)[torch.randperm(B, generator=g)] / max(1, sum(counts)) ** 0.5
    out = []
    for n in counts:
        x = (torch.randn(B, n, generator=g) * scale[:, None]).to(DTYPES[dtype])
        buf = torch.empty(B * n + offset, dtype=DTYPES[dtype], device=DEV)
        buf[offset:] = x.flatten().to(DEV)
        out.append(buf[offset:].view(B, n))
    return out


def _reference(Xs, C):
    x = [t.double().cpu() for t in Xs]
    n = sum((t * t).sum(1) for t in x)
    c = torch.where(n > 0, torch.clamp(C / n.sqrt(), max=1.0), torch.ones_like(n))
    return x, n, c


def _check_norms(got, n):
    assert torch.all((got.double().cpu() - n).abs() <= 64 * U * n), ((got.double().cpu() - n).abs() / n).max()


def _check_sums(got, x, c, before=0.0):
    B = x.shape[0]
    ref, most = (c[:, None] * x).sum(0), (c[:, None] * x).abs().sum(0)
    err = (got.double().cpu() - before - ref).abs()
    assert torch.all(err <= (B / 4 + 20 + 36) * U * (most + abs(before))), (err / (U * most + 1e-300)).max()


CASES = [(1, (1,)), (1, (7, 0, 8, 9)), (1, (4096, 4097, 100_003, 3)), (1, (1_000_003,)), (2, (1,) * 5), (3, (513, 1, 8191, 20_001)), (5, (12_289, 24)),
         (63, (512, 72)), (64, (511, 1030)), (65, (8, 3, 7)), (257, (1024,)), (600, (33, 256)), (1030, (17,))]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("B,counts", CASES)
def test_norms_sums_and_scaled(dp, B, counts, dtype, offset):
    C = 1.0
    Xs = _tensors(B, counts, dtype, 7 * B + len(counts), offset)
    x, n, c = _reference(Xs, C)
    sq = torch.zeros(B, device=DEV)
    dp.sqnorms_grads(Xs, sq)
    _check_norms(sq, n)
    bufs = [torch.full((k + 2 * offset,), 0.25, device=DEV) for k in counts]   # (not the alignment of the tensors)
    sums = [b[offset:offset + k] for b, k in zip(bufs, counts)]
    dp.clip_accumulate_grads(Xs, C, sq, sums)
    for s, t, b in zip(sums, x, bufs):
        _check_sums(s, t, c, 0.25)
        if offset:
            assert b[0] == 0.25 and b[-1] == 0.25   # neighbours stay as they were
    Ys = [torch.empty_like(t) for t in Xs]
    dp.clip_grads(Xs, C, sq, Ys)
    eps = torch.finfo(DTYPES[dtype]).eps / 2
    for y, t in zip(Ys, x):
        ref = c[:, None] * t
        assert torch.all((y.double().cpu() - ref).abs() <= (36 * U + eps * (1 + 36 * U)) * ref.abs())
        assert torch.equal(y.cpu()[c == 1], t.to(y.dtype)[c == 1])
    dp.clip_grads(Xs, C, sq, Xs)   # in place: the same bits
    for y, t in zip(Ys, Xs):
        assert torch.equal(y, t)
    dp.sync()


@pytest.mark.gpu
def test_many_tensors_and_other_calls_norms(dp):
    """More tensors than a launch holds, of both types in calls of their own, added to norms that are there already."""
    B, counts = 3, [(37 * k) % 1500 for k in range(300)]
    A, G = _tensors(B, counts, "f32", 1), _tensors(B, counts[::-1], "bf16", 2)
    _, n, _ = _reference(A + G, 1.0)
    sq = torch.full((B,), 0.5, device=DEV)
    dp.sqnorms_grads(A, sq)
    dp.sqnorms_grads(G, sq)
    _check_norms(sq, n + 0.5)
    c = torch.clamp(1.0 / (n + 0.5).sqrt(), max=1.0)
    for Xs in (A, G):
        sums = [torch.zeros(t.shape[1], device=DEV) for t in Xs]
        dp.clip_accumulate_grads(Xs, 1.0, sq, sums)
        for s, t in zip(sums, Xs):
            _check_sums(s, t.double().cpu(), c)


@pytest.mark.gpu
def test_small_workspace_gives_the_norms_too():
    import paper_2108_01624_amd as pkg

    B, counts = 4, (300_000, 50, 120_000, 9)
    Xs = _tensors(B, counts, "bf16", 3)
    _, n, _ = _reference(Xs, 1.0)
    for floats in (1, 2, 3, 40):
        with pkg.Context(workspace_bytes=4 * B * floats) as small:
            sq = torch.zeros(B, device=DEV)
            small.sqnorms_grads(Xs, sq)
            small.sync()
            # one piece a row: 300,000 / 1,024 additions in a thread
            assert torch.all((sq.double().cpu() - n).abs() <= 400 * U * n)
    with pkg.Context(workspace_bytes=4 * B - 4) as none:
        with pytest.raises(pkg.DpError) as e:
            none.sqnorms_grads(Xs, torch.zeros(B, device=DEV))
        assert e.value.status == -7


@pytest.mark.gpu
def test_sums_that_share_a_buffer(dp):
    """The same buffer for two tensors, and buffers that overlap in part: every tensor is added."""
    for B in (1, 3):
        Xs = _tensors(B, (5000, 5000, 3000), "f32", 4)
        x, n, c = _reference(Xs, 1.0)
        sq = torch.zeros(B, device=DEV)
        dp.sqnorms_grads(Xs, sq)
        S = torch.zeros(6000, device=DEV)
        dp.clip_accumulate_grads(Xs, 1.0, sq, [S[:5000], S[:5000], S[3000:]])
        ref, most = torch.zeros(6000, dtype=torch.float64), torch.zeros(6000, dtype=torch.float64)
        for t, o in zip(x, (0, 0, 3000)):
            ref[o:o + t.shape[1]] += (c[:, None] * t).sum(0)
            most[o:o + t.shape[1]] += (c[:, None] * t).abs().sum(0)
        assert torch.all((S.double().cpu() - ref).abs() <= 64 * U * most)


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("B", [1, 3])
def test_norms_that_are_not_finite_are_reported(dp, B, bad):
    import paper_2108_01624_amd as pkg

    Xs = _tensors(B, (5000, 10), "f32", 5)
    Xs[0][B - 1, 4321] = bad
    sq = torch.zeros(B, device=DEV)
    dp.sqnorms_grads(Xs, sq)
    dp.sync()
    S, Y = [torch.zeros(5000, device=DEV), torch.zeros(10, device=DEV)], [torch.zeros_like(t) for t in Xs]
    for call in (lambda: dp.clip_accumulate_grads(Xs, 1.0, sq, S), lambda: dp.clip_grads(Xs, 1.0, sq, Y)):
        call()
        with pytest.raises(pkg.DpError) as e:
            dp.sync()
        assert e.value.status == -5
    assert all(torch.isnan(s).all() for s in S)
    for y, t in zip(Y, Xs):
        assert torch.isnan(y[B - 1]).all() and not torch.isnan(y[:B - 1]).any()


@pytest.mark.gpu
def test_zero_and_denormal_gradients(dp):
    Xs = [torch.zeros(2, 1000, device=DEV)]
    Xs[0][1] = 1e-30   # its square is zero in fp32: the factor is one
    sq, S = torch.zeros(2, device=DEV), torch.zeros(1000, device=DEV)
    dp.sqnorms_grads(Xs, sq)
    dp.clip_accumulate_grads(Xs, 1.0, sq, [S])
    dp.sync()
    assert not sq.any() and torch.equal(S, Xs[0][1])


def test_refusals():
    """Argument checks of the library: they come before anything touches the context's stream, so a block of zeros stands in for a context."""
    import paper_2108_01624_amd as pkg

    lib = pkg.load_library()
    ctx = ctypes.create_string_buffer(1 << 14)
    keep = np.zeros(64, dtype=np.float32)
    p = keep.ctypes.data
    tab = lambda *a: (ctypes.c_void_p * len(a))(*a)
    cnt = lambda *a: (ctypes.c_uint64 * len(a))(*a)
    F, H = pkg.DP_F32, pkg.DP_BF16
    assert lib.dp_sqnorms_grads(None, 1, tab(p), cnt(1), F, 1, p) == -1
    norms = lambda n=1, X=tab(p), c=cnt(4), dt=F, B=1, sq=p: lib.dp_sqnorms_grads(ctx, n, X, c, dt, B, sq)
    assert norms(n=0) == 0 and norms(B=0) == 0
    assert norms(dt=2) == -3 and norms(n=-1) == -2 and norms(B=-1) == -2 and norms(sq=None) == -1 and norms(sq=p + 2) == -4
    assert norms(X=None) == -1 and norms(c=None) == -1 and norms(X=tab(None)) == -1 and norms(X=tab(p + 2)) == -4 and norms(X=tab(p + 1), dt=H) == -4
    assert norms(c=cnt(1 << 60)) == -2 and norms(c=cnt((1 << 31) + 1), B=2) == -2
    sums = lambda n=1, X=tab(p), c=cnt(4), dt=F, B=1, C=1.0, sq=p, S=tab(p): lib.dp_clip_accumulate_grads(ctx, n, X, c, dt, B, C, sq, S)
    assert sums(S=None) == -1 and sums(S=tab(None)) == -1 and sums(S=tab(p + 2)) == -4 and sums(C=0.0) == -5 and sums(C=float("nan")) == -5
    assert sums(dt=H, S=tab(p + 2)) == -4 and sums(B=0) == 0 and sums(n=0) == 0 and sums(n=0, S=None, X=None, c=None) == 0
    scale = lambda n=1, X=tab(p), c=cnt(4), dt=F, B=1, C=1.0, sq=p, Y=tab(p): lib.dp_clip_grads(ctx, n, X, c, dt, B, C, sq, Y)
    assert scale(Y=None) == -1 and scale(Y=tab(None)) == -1 and scale(Y=tab(p + 2)) == -4 and scale(dt=H, Y=tab(p + 1)) == -4 and scale(C=-1.0) == -5


def test_refusals_of_tensors():
    import paper_2108_01624_amd as pkg

    if torch.cuda.is_available():
        pytest.skip("on the CPU, where no call could touch memory")
    pkg.load_library()
    ctx = ctypes.addressof(ctypes.create_string_buffer(1 << 14))
    sq, x = torch.zeros(2), torch.zeros(2, 6)
    for Xs, out in (([torch.zeros(3, 6)], [torch.zeros(6)]), ([torch.zeros(6, 2).t()], [torch.zeros(6)]), ([x, x.bfloat16()], [torch.zeros(6)] * 2),
                    ([x], [torch.zeros(7)]), ([x], [torch.zeros(6), torch.zeros(6)]), ([x], [torch.zeros(12)[::2]])):
        with pytest.raises((ValueError, TypeError)):
            pkg.dp_clip_accumulate_grads(ctx, Xs, 1.0, sq, out)
    for Y in (torch.zeros(2, 6, dtype=torch.bfloat16), torch.zeros(2, 5), torch.zeros(6, 2).t()):
        with pytest.raises(ValueError):
            pkg.dp_clip_grads(ctx, [x], 1.0, sq, [Y])
    with pytest.raises(TypeError):
        pkg.dp_sqnorms_grads(ctx, [x.half()], sq)
    with pytest.raises(TypeError):
        pkg.dp_sqnorms_grads(ctx, [x], sq.double())


def test_refusals_of_outputs_that_overlap():
    """Outputs over inputs, norms or each other: refused before anything is launched, wherever in the call the two tensors stand.  What is allowed goes
    on to its launch, which fails for want of a GPU (-8)."""
    import paper_2108_01624_amd as pkg

    if torch.cuda.is_available():
        pytest.skip("on the CPU, where no call could touch memory")
    lib = pkg.load_library()
    ctx = ctypes.create_string_buffer(1 << 14)
    keep = np.zeros(1 << 16, dtype=np.float32)
    p = keep.ctypes.data
    sq = p + 4 * 60000
    tab = lambda a: (ctypes.c_void_p * len(a))(*a)
    cnt = lambda a: (ctypes.c_uint64 * len(a))(*a)
    F, H = pkg.DP_F32, pkg.DP_BF16

    def scale(X, Y, counts, B=2, dt=F, sq=sq):
        return lib.dp_clip_grads(ctx, len(X), tab(X), cnt(counts), dt, B, 1.0, sq, tab(Y))

    def sums(X, S, counts, B=2, dt=F, sq=sq):
        return lib.dp_clip_accumulate_grads(ctx, len(X), tab(X), cnt(counts), dt, B, 1.0, sq, tab(S))

    at = lambda *floats: [p + 4 * f for f in floats]
    for order in (1, -1):
        o = lambda a: a[::order]
        # 40 tensors of 2 x 10 numbers: X at 0, 20, ..., Y behind them
        X, Y = at(*range(0, 800, 20)), at(*range(800, 1600, 20))
        assert scale(o(X), o(Y), [10] * 40) == -8 and scale(o(X), o(X), [10] * 40) == -8 and scale(X, X[:20] + Y[20:], [10] * 40) == -8
        assert scale(o(Y), o(X), [10] * 40) == -8 and sums(o(X), o(Y), [10] * 40) == -8 and sums(X, Y[::-1], [10] * 40) == -8
        assert scale(o(X[:-1] + X[:1]), o(X[:-1] + X[:1]), [10] * 40) == -5        # a tensor listed twice, in place
        assert scale(X, o(Y[:-1] + Y[:1]), [10] * 40) == -5                        # one output for two
        assert scale(X, o(Y[:7] + [Y[7] + 4] + Y[8:]), [10] * 40) == -5            # an output that reaches into the next
        assert scale(X, o(Y[:7] + [X[39]] + Y[8:]), [10] * 40) == -5               # ... or over another tensor's input
        assert scale(o(X), o([X[0] + 4] + Y[1:]), [10] * 40) == -5                 # in place, but for one number
        assert scale(X, X[1:] + [X[0]], [10] * 40) == -5
        assert sums(X, o(Y[:39] + [X[3] + 76]), [10] * 40) == -5                   # the last number of an input
        assert sums(X, o(Y[:39] + [X[3] - 36]), [10] * 40) == -5                   # the first
        assert sums(X[1:], o(Y[:38] + [X[0]]), [10] * 39) == -8                    # in front of all of them
        assert sums(X, o(Y[:39] + Y[:1]), [10] * 40) == -8                         # sums may share
        assert scale(X, Y, [10] * 39 + [0]) == -8 and scale(X, o(Y[:39] + X[3:4]), o([10] * 39 + [0])) == -8   # (a tensor of no elements has no place)
        assert scale(X, o(Y), [10] * 40, sq=Y[5] + 76) == -5 and sums(X, o(Y), [10] * 40, sq=Y[5] + 36) == -5 and scale(o(X), o(X), [10] * 40, sq=X[5]) == -5
        assert scale(X, o(Y), [10] * 40, sq=Y[39] + 80) == -8 and sums(X, o(Y), [10] * 40, sq=X[7]) == -8
    # bf16 ranges are half as long, sums are not
    assert scale(at(0, 10), at(20, 30), [10, 10], dt=H) == -8 and scale(at(0, 10), at(19, 30), [10, 10], dt=H) == -5
    assert sums(at(0, 10), at(20, 30), [10, 10], dt=H) == -8 and sums(at(0, 10), at(19, 30), [10, 10], dt=H) == -5 and sums(at(20), at(11), [10], dt=H) == -5
    assert sums(at(20), at(10), [10], dt=H) == -8
    norms = lambda sq, dt=F, B=2, counts=(10, 10): lib.dp_sqnorms_grads(ctx, 2, tab(at(0, 100)), cnt(counts), dt, B, sq)
    assert norms(p + 76) == -5 and norms(p + 4 * 99) == -5 and norms(p + 4 * 119) == -5 and norms(p + 40, dt=H, counts=(10, 0)) != -5
    assert norms(p + 80) != -5 and norms(p + 4 * 98) != -5 and norms(p + 4 * 120) != -5 and norms(p + 4 * 100, counts=(10, 0)) != -5


@pytest.mark.gpu
def test_a_tied_tensor_in_place_is_refused_and_left_alone(dp):
    import paper_2108_01624_amd as pkg

    Xs = _tensors(3, (5000, 700), "bf16", 11)
    before = [t.clone() for t in Xs]
    sq = torch.full((3,), 100.0, device=DEV)
    for outs in ([Xs[0], Xs[1], Xs[0]], [torch.empty_like(Xs[0]), Xs[0].flatten()[:2100].view(3, 700), Xs[0]]):
        with pytest.raises(pkg.DpError) as e:
            dp.clip_grads([Xs[0], Xs[1], Xs[0]], 1.0, sq, outs)
        assert e.value.status == -5
    buf = torch.zeros(5000 + 700, device=DEV)
    with pytest.raises(pkg.DpError) as e:
        dp.clip_accumulate_grads([buf[:5000].view(1, 5000), torch.zeros(1, 700, device=DEV)], 1.0, sq[:1], [torch.zeros(5000, device=DEV), buf[4999:-1]])
    assert e.value.status == -5
    dp.sync()
    assert all(torch.equal(a, b) for a, b in zip(Xs, before)) and not buf.any()
    # what does not meet is taken: every second tensor of a buffer in place, the others beside their inputs
    flat = torch.randn(8, 3, 1000, device=DEV)
    X = list(flat)
    Y = [x if k % 2 else torch.empty_like(x) for k, x in enumerate(X)]
    want = [x * 0.1 for x in X]
    dp.clip_grads(X, 1.0, sq, Y)
    dp.sync()
    assert all(((y - w).abs() <= 40 * U * w.abs()).all() for y, w in zip(Y, want))
