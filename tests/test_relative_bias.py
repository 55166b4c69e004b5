"""The relative position bias by buckets and every example's gradient of its table.

The bias is a table entry rounded once: equal to torch's rounding of it.  A gradient is a sum in fp32 in some fixed order: with u = 2^-24 it is
off by at most u times its additions times the sum of the terms' magnitudes.  A term passes at most L Tq additions of its diagonal in a thread, those
of up to 256 groups, (Tq + Tk) / 64 in a lane of its bucket's wave, 6 over the lanes and those of the parts of a plane (up to Tq / 8)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from gpu_util import DEV

U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _bucket(rel, starts, both):
    """Bucket numbers by plain comparison, for a table of distances."""
    dist = rel.abs() if both else (-rel).clamp(min=0)
    b = torch.zeros_like(rel)
    for j, s in enumerate(starts):
        b[dist >= s] = j
    return torch.where(rel > 0, b + len(starts), b) if both else b


def _rel(Tq, Tk):
    return torch.arange(Tk)[None, :] - (torch.arange(Tq) + Tk - Tq)[:, None]


def _customary(n, reach):
    """starts of the customary buckets by whole numbers."""
    e, out = n // 2, list(range(n // 2))
    for j in range(n - e):
        d = e
        while d ** (n - e) * e ** j < reach ** j * e ** (n - e):
            d += 1
        out.append(d)
    return out


@pytest.mark.parametrize("n,reach", [(2, 2), (3, 5), (4, 4), (8, 20), (16, 128), (32, 128), (16, 8192), (33, 1000), (64, 65), (128, 512)])
def test_customary_buckets(n, reach):
    import paper_2108_01624_amd as pkg

    starts = pkg.dp_relative_buckets(n, reach)
    assert starts == _customary(n, reach)
    if (n, reach) == (16, 128):   # the halves of an octave
        assert starts == [0, 1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 23, 32, 46, 64, 91]


def test_customary_buckets_refusals():
    import paper_2108_01624_amd as pkg

    for n, reach in ((1, 8), (0, 8), (-3, 8), (129, 1000), (16, 8), (16, 0), (16, (1 << 30) + 1)):
        with pytest.raises(pkg.DpError) as e:
            pkg.dp_relative_buckets(n, reach)
        assert e.value.status == -5
    assert len(pkg.dp_relative_buckets(16, 1 << 30)) == 16


STARTS = {"t16": _customary(16, 128), "one": [0], "gaps": [0, 0, 3, 3, 9, 1000], "n128": list(range(128))}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("starts,both", [("t16", True), ("t16", False), ("one", True), ("gaps", False), ("gaps", True), ("n128", True)])
@pytest.mark.parametrize("H,Tq,Tk", [(1, 1, 1), (3, 1, 2), (2, 1, 4097), (5, 33, 33), (2, 64, 64), (3, 7, 129), (2, 130, 2100), (16, 40, 41)])
def test_bias(dp, dtype, starts, both, H, Tq, Tk):
    s = STARTS[starts]
    table = torch.randn(len(s) * (2 if both else 1), H, generator=torch.Generator().manual_seed(H + Tk))
    out = torch.full((H * Tq * Tk + 2,), 7.0, dtype=DTYPES[dtype], device=DEV)
    bias = out[1:-1].view(H, Tq, Tk)   # (aligned to an element only)
    dp.relative_bias(table.to(DEV), s, both, bias)
    dp.sync()
    assert torch.equal(bias.cpu(), table[_bucket(_rel(Tq, Tk), s, both)].permute(2, 0, 1).to(DTYPES[dtype]))
    assert out[0] == 7 and out[-1] == 7


def _grads_reference(dS, s, both, lengths, causal):
    B, H, Tq, Tk = dS[0].shape
    ok = torch.ones(B, 1, Tq, Tk, dtype=torch.bool)
    pos = torch.arange(Tq) + Tk - Tq
    if lengths is not None:
        ok &= (pos[None, :, None] < lengths[:, None, None])[:, None] & (torch.arange(Tk)[None, None, :] < lengths[:, None, None])[:, None]
    if causal:
        ok &= _rel(Tq, Tk) <= 0
    idx = _bucket(_rel(Tq, Tk), s, both).flatten()
    n = len(s) * (2 if both else 1)
    total, most = (torch.zeros(B, H, n, dtype=torch.float64) for _ in range(2))
    for x in dS:
        x = torch.where(ok, x.double().cpu(), torch.zeros((), dtype=torch.float64)).flatten(2)
        total.index_add_(2, idx, x)
        most.index_add_(2, idx, x.abs())
    return total.transpose(1, 2), most.transpose(1, 2)


def _check_grads(got, dS, s, both, lengths=None, causal=False):
    ref, most = _grads_reference(dS, s, both, lengths, causal)
    Tq, Tk = dS[0].shape[2:]
    steps = len(dS) * Tq + 256 + (Tq + Tk) / 64 + 8 + Tq / 8
    err = (got.double().cpu() - ref).abs()
    assert torch.all(err <= steps * U * most), (err / (U * most + 1e-300)).max()


def _scores(L, B, H, Tq, Tk, dtype, seed, offset=0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for _ in range(L):
        buf = torch.empty(B * H * Tq * Tk + offset, dtype=DTYPES[dtype], device=DEV)
        buf[offset:] = torch.randn(B * H * Tq * Tk, generator=g).to(DEV)
        out.append(buf[offset:].view(B, H, Tq, Tk))
    return out


SHAPES = [(1, 1, 1, 1, 1), (2, 3, 2, 1, 9), (1, 2, 1, 1, 700), (3, 2, 2, 7, 7), (24, 2, 2, 8, 8), (1, 3, 5, 9, 17), (2, 1, 3, 63, 63), (1, 4, 2, 64, 64),
          (2, 2, 2, 65, 130), (1, 1, 1, 129, 129), (3, 1, 1, 255, 257), (1, 300, 4, 20, 20), (1, 1, 1, 40, 2060), (130, 1, 2, 5, 6)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,offset", [("bf16", 0), ("bf16", 1), ("f32", 0), ("f32", 1)])
@pytest.mark.parametrize("L,B,H,Tq,Tk", SHAPES)
def test_grads(dp, L, B, H, Tq, Tk, dtype, offset):
    dS = _scores(L, B, H, Tq, Tk, dtype, L + Tq + Tk, offset)
    for starts, both, causal in (("t16", True, False), ("t16", False, True), ("gaps", False, False), ("n128", True, True)):
        s = STARTS[starts]
        buf = torch.full((B * len(s) * (2 if both else 1) * H + 2,), 7.0, device=DEV)
        grads = buf[1:-1].view(B, len(s) * (2 if both else 1), H)
        dp.relative_bias_grads(dS, s, both, grads, causal=causal)
        dp.sync()
        _check_grads(grads, dS, s, both, None, causal)
        assert buf[0] == 7 and buf[-1] == 7


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Tq,Tk", [(1, 13), (13, 13), (64, 64), (50, 77), (131, 131)])
@pytest.mark.parametrize("causal", [False, True])
def test_grads_of_a_padded_batch(dp, dtype, Tq, Tk, causal):
    """Lengths from none to all (and beyond both ends), with NaN and infinities in every place that does not count."""
    lengths = torch.tensor([0, Tk, 1, Tk - 1, Tk // 2, Tk - Tq, -3, Tk + 5, min(Tk, 9)], dtype=torch.int32)
    B, H = len(lengths), 2
    dS = _scores(2, B, H, Tq, Tk, dtype, Tk)
    pos, key, n = torch.arange(Tq) + Tk - Tq, torch.arange(Tk), lengths[:, None, None]
    out = ~((pos[None, :, None] < n) & (key[None, None, :] < n))[:, None].expand(B, H, Tq, Tk)
    if causal:
        out = out | (_rel(Tq, Tk) > 0)
    dS[0][out.to(DEV)] = float("nan")
    dS[1][out.to(DEV)] = float("inf")
    s = STARTS["t16"]
    grads = torch.empty(B, 2 * len(s), H, device=DEV)
    dp.relative_bias_grads(dS, s, True, grads, lengths=lengths.to(DEV), causal=causal)
    dp.sync()
    _check_grads(grads, dS, s, True, lengths, causal)
    assert not grads[0].any() and not grads[6].any()


@pytest.mark.gpu
def test_grads_longest_line_and_small_workspace():
    import paper_2108_01624_amd as pkg

    s = STARTS["t16"]
    with pkg.Context() as ctx:
        dS = _scores(1, 1, 1, 3, 32765, "bf16", 1)   # Tq + Tk = 32,768
        grads = torch.empty(1, 32, 1, device=DEV)
        ctx.relative_bias_grads(dS, s, True, grads)
        ctx.sync()
        _check_grads(grads, dS, s, True)
        with pytest.raises(pkg.DpError) as e:
            ctx.relative_bias_grads(_scores(1, 1, 1, 4, 32765, "bf16", 1), s, True, grads)
        assert e.value.status == -2
    dS = _scores(2, 2, 1, 300, 300, "f32", 2)
    for floats in (1, 2 * 32 * 3, 1 << 16):   # no room for parts, room for three, for all
        with pkg.Context(workspace_bytes=4 * floats) as small:
            grads = torch.empty(2, 32, 1, device=DEV)
            small.relative_bias_grads(dS, s, True, grads)
            small.sync()
            _check_grads(grads, dS, s, True)
    many = [dS[0]] * 129   # two launches, whose parts have to fit
    with pkg.Context(workspace_bytes=4) as none:
        with pytest.raises(pkg.DpError) as e:
            none.relative_bias_grads(many, s, True, grads)
        assert e.value.status == -7


@pytest.mark.gpu
def test_gradient_is_that_of_the_bias(dp):
    """<grads, D> is the change of sum(dS * bias) along a change D of the table: the bias is linear in its table."""
    s, H, Tq, Tk = STARTS["t16"], 3, 50, 70
    dS = _scores(1, 1, H, Tq, Tk, "f32", 3)
    grads, bias = torch.empty(1, 2 * len(s), H, device=DEV), torch.empty(H, Tq, Tk, device=DEV)
    dp.relative_bias_grads(dS, s, True, grads)
    for b in range(0, 2 * len(s), 5):
        D = torch.zeros(2 * len(s), H, device=DEV)
        D[b] = 1.0
        dp.relative_bias(D, s, True, bias)
        terms = (dS[0][0].double() * bias.double())
        assert torch.all((terms.sum((1, 2)) - grads[0, b].double()).abs() <= 400 * U * terms.abs().sum((1, 2)))
    dp.sync()


@pytest.mark.gpu
def test_no_layers_and_no_queries_write_zeros(dp):
    import paper_2108_01624_amd as pkg

    grads = torch.ones(3, 32, 2, device=DEV)
    dp.relative_bias_grads([torch.empty(3, 2, 0, 5, device=DEV)], STARTS["t16"], True, grads)
    assert not grads.any()
    grads.fill_(1)
    starts = (ctypes.c_int32 * 16)(*STARTS["t16"])
    assert pkg.load_library().dp_relative_bias_grads(dp.handle, 0, None, pkg.DP_F32, None, 0, 16, starts, 1, 3, 2, 5, 5, grads.data_ptr()) == 0
    dp.sync()
    assert not grads.any()


def test_refusals():
    """Argument checks of the library: they come before anything touches the context's stream, so a block of zeros stands in for a context."""
    import paper_2108_01624_amd as pkg

    lib = pkg.load_library()
    ctx = ctypes.create_string_buffer(1 << 14)
    keep = np.zeros(64, dtype=np.float32)
    p = keep.ctypes.data
    st = lambda *a: (ctypes.c_int32 * len(a))(*a)
    F, BF = pkg.DP_F32, pkg.DP_BF16
    assert lib.dp_relative_bias(None, p, 1, st(0), 0, 1, 1, 1, F, p) == -1
    bias = lambda t=p, n=2, s=st(0, 1), H=1, Tq=2, Tk=2, dt=F, out=p: lib.dp_relative_bias(ctx, t, n, s, 1, H, Tq, Tk, dt, out)
    assert bias(H=0) == 0 and bias(Tq=0) == 0
    assert bias(t=None) == -1 and bias(out=None) == -1 and bias(s=None) == -1 and bias(t=p + 2) == -4 and bias(out=p + 2) == -4 and bias(out=p + 1, dt=BF) == -4
    assert bias(dt=7) == -3 and bias(n=0) == -2 and bias(n=129) == -2 and bias(Tq=3) == -2 and bias(Tq=-1) == -2 and bias(H=-1) == -2 and bias(Tk=(1 << 30) + 1) == -2
    for s in (st(1, 2), st(0, -1), st(-1, 0), st(0, (1 << 30) + 1)):
        assert bias(s=s) == -5
    assert bias(n=3, s=st(0, 5, 4)) == -5
    tab = lambda *a: (ctypes.c_void_p * len(a))(*a)
    grads = lambda L=1, x=tab(p), dt=F, ln=None, n=2, s=st(0, 1), B=1, H=1, Tq=2, Tk=2, g=p: lib.dp_relative_bias_grads(ctx, L, x, dt, ln, 0, n, s, 1, B, H, Tq, Tk, g)
    assert grads(B=0) == 0 and grads(H=0) == 0
    assert grads(x=None) == -1 and grads(x=tab(None)) == -1 and grads(g=None) == -1 and grads(x=tab(p + 2)) == -4 and grads(x=tab(p + 1), dt=BF) == -4 and grads(g=p + 1) == -4
    assert grads(ln=p + 2) == -4 and grads(L=-1) == -2 and grads(B=-1) == -2 and grads(Tq=16385, Tk=16384) == -2 and grads(Tq=16385, Tk=16385) == -2 and grads(s=st(0, -5)) == -5


def test_refusals_of_tensors():
    import paper_2108_01624_amd as pkg

    if torch.cuda.is_available():
        pytest.skip("on the CPU, where no call could touch memory")
    pkg.load_library()
    ctx = ctypes.addressof(ctypes.create_string_buffer(1 << 14))
    s = [0, 1, 2]
    for table, both, bias in ((torch.zeros(3, 2), True, torch.zeros(2, 4, 4)), (torch.zeros(6, 3), True, torch.zeros(2, 4, 4)), (torch.zeros(2, 3).t(), False, torch.zeros(2, 4, 4)),
                              (torch.zeros(3, 2), False, torch.zeros(2, 4, 8)[..., ::2]), (torch.zeros(3, 2).double(), False, torch.zeros(2, 4, 4)),
                              (torch.zeros(3, 2), False, torch.zeros(2, 4, 4).half())):
        with pytest.raises((ValueError, TypeError)):
            pkg.dp_relative_bias(ctx, table, s, both, bias)
    x, g = torch.zeros(2, 2, 4, 4), torch.zeros(2, 6, 2)
    for dS, grads, lengths in (([x, x.bfloat16()], g, None), ([x, torch.zeros(2, 2, 4, 5)], g, None), ([x.transpose(2, 3)], g, None), ([x], torch.zeros(2, 3, 2), None),
                               ([x], g, torch.zeros(3, dtype=torch.int32)), ([x], g, torch.zeros(2)), ([x], torch.zeros(2, 2, 6).transpose(1, 2), None)):
        with pytest.raises((ValueError, TypeError)):
            pkg.dp_relative_bias_grads(ctx, dS, s, True, grads, lengths=lengths)


def _additions(L, Tq, Tk, parts):
    """Additions on the longest path of a score's gradient into its bucket: one per row and layer in a thread; a diagonal's four sums (of two bands,
    before and after their step over) of at most 256 groups of threads, which share rows of blocks and layers; sixteen lanes to a bucket's diagonals
    (those of a far band: 15, one per 256 blocks of a row, 6 over the lanes and 8 waves); the parts of a plane, sixteen lanes as well."""
    return L * Tq + 4 * min(256, L * (Tq // 8 + 1)) + max((Tq + Tk) / 16 + 4, 15 + Tk / 2048 + 14) + 8 + parts / 16 + 5


def _check_sums(got, dS, s, both, lengths, causal):
    ref, most = _grads_reference(dS, s, both, lengths, causal)
    Tq, Tk = dS[0].shape[2:]
    err = (got.double().cpu() - ref).abs()
    assert torch.all(err <= _additions(len(dS), Tq, Tk, Tq / 8 + 1) * U * most), (err / (U * most + 1e-300)).max()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("both,causal", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("Tq,Tk,last", [(3, 32765, 30000), (3, 32765, 1 << 30), (600, 9000, 8700), (2, 8750, 8749), (2, 8700, 8699)])
def test_grads_whose_diagonals_fill_the_local_memory(dp, Tq, Tk, last, both, causal, dtype):
    """Last starts so far away that most of the Tq + Tk - 1 diagonals are taken apart: up to 158 KiB of a CU's memory, below and above 64."""
    starts = [0, 1, 2, 3, 50, 51, 700, last // 2, last - 1, last]
    dS = _scores(1, 2, 1, Tq, Tk, dtype, Tq + Tk)
    grads = torch.empty(2, len(starts) * (2 if both else 1), 1, device=DEV)
    dp.relative_bias_grads(dS, starts, both, grads, causal=causal)
    dp.sync()
    _check_sums(grads, dS, starts, both, None, causal)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("starts,both", [("t16", False), ("far", True)])
@pytest.mark.parametrize("T", [2040, 2041, 2049, 2100])
def test_grads_of_long_squares_under_a_causal_mask(dp, T, starts, both, padded, dtype):
    """Rows of blocks, two of which are a step, around what the threads of a workgroup hold at a time (256 blocks), with NaN and infinities behind
    the lengths and the mask."""
    s = dict(STARTS, far=[0, 1, 5, 16, 900, 2030])[starts]
    lengths = torch.tensor([T, T - 9, 1030], dtype=torch.int32) if padded else None
    B = 3 if padded else 1
    dS = _scores(2, B, 1, T, T, dtype, T)
    out = (_rel(T, T) > 0).expand(B, 1, T, T)
    if padded:
        pos = torch.arange(T)
        out = out | ~((pos[None, :, None] < lengths[:, None, None]) & (pos[None, None, :] < lengths[:, None, None]))[:, None]
    dS[0][out.to(DEV)] = float("nan")
    dS[1][out.to(DEV)] = float("inf")
    grads = torch.empty(B, len(s) * (2 if both else 1), 1, device=DEV)
    dp.relative_bias_grads(dS, s, both, grads, lengths=None if lengths is None else lengths.to(DEV), causal=True)
    dp.sync()
    _check_sums(grads, dS, s, both, lengths, True)


def test_refusals_of_outputs_that_overlap():
    """What is written over what is read: refused before anything is launched.  What is allowed goes on to its launch, which fails for want of a GPU (-8)."""
    import paper_2108_01624_amd as pkg

    if torch.cuda.is_available():
        pytest.skip("on the CPU, where no call could touch memory")
    lib = pkg.load_library()
    ctx = ctypes.create_string_buffer(1 << 14)
    keep = np.zeros(2000, dtype=np.float32)
    at = lambda k: keep.ctypes.data + 4 * k
    st = (ctypes.c_int32 * 2)(0, 1)
    F, BF, H, Tq, Tk, B = pkg.DP_F32, pkg.DP_BF16, 3, 4, 5, 2
    bias = lambda t, out, both=1, dt=F: lib.dp_relative_bias(ctx, t, 2, st, both, H, Tq, Tk, dt, out)
    # a table of 12 numbers (6 without buckets behind the query), a bias of 60
    assert bias(at(0), at(12)) == -8 and bias(at(0), at(11)) == -5 and bias(at(0), at(6), both=0) == -8 and bias(at(0), at(5), both=0) == -5
    assert bias(at(60), at(0)) == -8 and bias(at(59), at(0)) == -5 and bias(at(30), at(0), dt=BF) == -8 and bias(at(29), at(0), dt=BF) == -5
    # 24 gradients, scores of 120 numbers, two lengths
    def grads(g, x, ln=None, dt=F):
        return lib.dp_relative_bias_grads(ctx, len(x), (ctypes.c_void_p * len(x))(*x), dt, ln, 0, 2, st, 1, B, H, Tq, Tk, g)

    x = [at(k) for k in (0, 120, 240)]
    assert grads(at(360), x) == -8 and grads(at(359), x) == -5 and grads(at(120), x) == -5 and grads(at(120), x[::2]) == -8 and grads(at(97), x[1:]) == -5
    assert grads(at(96), x[1:]) == -8 and grads(at(60), x[:1], dt=BF) == -8 and grads(at(59), x[:1], dt=BF) == -5
    assert grads(at(360), x, ln=at(384)) == -8 and grads(at(360), x, ln=at(383)) == -5 and grads(at(360), x, ln=at(359)) == -5 and grads(at(400), x, ln=at(398)) == -8


def test_numbers_beyond_32_bits_are_refused():
    """... and not cut down to what is left of them, in the functions as in the methods of a context (which leave such numbers to the functions)."""
    import paper_2108_01624_amd as pkg

    if torch.cuda.is_available():
        pytest.skip("on the CPU, where no call could touch memory")
    pkg.load_library()
    for n, reach in ((16, (1 << 32) + 128), (16, 128 - (1 << 32)), ((1 << 32) + 16, 128), (16 - (1 << 32), 128), (-1, 128), (16, 1 << 80)):
        with pytest.raises(pkg.DpError) as e:
            pkg.dp_relative_buckets(n, reach)
        assert e.value.status == -5
    block = ctypes.create_string_buffer(1 << 14)
    ctx = object.__new__(pkg.Context)
    ctx.handle = ctypes.addressof(block)
    table, bias, dS, grads = torch.zeros(3, 2), torch.zeros(2, 4, 4), torch.zeros(2, 2, 4, 4), torch.zeros(2, 3, 2)
    for s in ([0, 1, (1 << 32) + 5], [0, 1 - (1 << 32), 5], [1 << 32, 1, 5], [0, 1, 1 << 70], [0, 1, (1 << 30) + 1]):
        for call in (lambda: pkg.dp_relative_bias(ctx.handle, table, s, False, bias), lambda: ctx.relative_bias(table, s, False, bias),
                     lambda: pkg.dp_relative_bias_grads(ctx.handle, [dS], s, False, grads), lambda: ctx.relative_bias_grads([dS], s, False, grads)):
            with pytest.raises(pkg.DpError) as e:
                call()
            assert e.value.status == -5
    table, s, long = torch.zeros(3, 0), [0, 1, 2], (1 << 32) + 8   # (no heads: nothing to allocate)
    for call in (lambda: ctx.relative_bias(table, s, False, torch.zeros(0, 4, long)), lambda: ctx.relative_bias(table, s, False, torch.zeros(0, long, 4)),
                 lambda: ctx.relative_bias_grads([torch.zeros(2, 0, 4, long)], s, False, torch.zeros(2, 3, 0))):
        with pytest.raises(pkg.DpError) as e:
            call()
        assert e.value.status == -2
    ctx.handle = None


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Tq,Tk", [(700, 700), (333, 1500), (1, 5000)])
@pytest.mark.parametrize("causal", [False, True])
def test_grads_of_a_padded_batch_of_long_examples(dp, dtype, Tq, Tk, causal):
    """Planes that several workgroups share, of which short examples leave some without work; NaN and infinities in every place that does not count."""
    lengths = torch.tensor([Tk, 0, Tk - 3, Tk // 2 + 1, Tk - Tq, Tk - Tq + 1], dtype=torch.int32)
    B, H = len(lengths), 2
    dS = _scores(3, B, H, Tq, Tk, dtype, Tk)
    pos, key, n = torch.arange(Tq) + Tk - Tq, torch.arange(Tk), lengths[:, None, None]
    out = ~((pos[None, :, None] < n) & (key[None, None, :] < n))[:, None].expand(B, H, Tq, Tk)
    if causal:
        out = out | (_rel(Tq, Tk) > 0)
    for x, v in zip(dS, (float("nan"), float("inf"), -float("inf"))):
        x[out.to(DEV)] = v
    for s, both in ((STARTS["t16"], True), ([0, 2, 30, 600], True), (STARTS["n128"], False)):
        grads = torch.full((B, len(s) * (2 if both else 1), H), 5.0, device=DEV)
        dp.relative_bias_grads(dS, s, both, grads, lengths=lengths.to(DEV), causal=causal)
        dp.sync()
        _check_sums(grads, dS, s, both, lengths, causal)


@pytest.mark.gpu
def test_grads_of_long_lines_replay_from_a_graph():
    """More local memory than a launch has without asking: the request may be made while a graph is recorded."""
    import paper_2108_01624_amd as pkg

    s = [0, 1, 30, 11000]
    x = [_scores(1, 2, 1, 5, 12000, "bf16", k)[0] for k in range(3)]
    side = torch.cuda.Stream(device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        ctx = pkg.Context()
        dS, grads = x[0].clone(), torch.empty(2, 8, 1, device=DEV)
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            ctx.relative_bias_grads([dS], s, True, grads)
    for k in (1, 0, 2, 2):
        with torch.cuda.stream(side):
            dS.copy_(x[k])
            grads.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ctx.sync()
        _check_sums(grads, [x[k]], s, True, None, False)
        eager = torch.empty_like(grads)
        ctx.relative_bias_grads([x[k]], s, True, eager)
        ctx.sync()
        assert torch.equal(eager, grads)
    del graph
    ctx.close()


@pytest.mark.gpu
def test_a_table_that_no_layer_uses_has_no_gradient(dp):
    import paper_2108_01624_amd as pkg

    s = STARTS["t16"]
    for both in (False, True):
        for call in (dp.relative_bias_grads, lambda *a: pkg.dp_relative_bias_grads(dp.handle, *a)):
            grads = torch.ones(3, 16 * (1 + both), 2, device=DEV)
            call([], s, both, grads)
            dp.sync()
            assert not grads.any()
    for wrong in (torch.ones(3, 15, 2, device=DEV), torch.ones(16, 2, device=DEV), torch.ones(3, 16, 2, device=DEV).bfloat16()):
        with pytest.raises((ValueError, TypeError)):
            dp.relative_bias_grads([], s, False, wrong)
    dp.sync()
