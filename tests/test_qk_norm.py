"""Norms of queries and keys with the rotation by position, and their backward, against the definition in 64 bits.

Tolerances, u = 2^-24.  The mean square adds D non-negative terms over at most 8 + 6 additions, so r is off by half of that and four more roundings;
a rotated number is a difference of two products: off by its roundings times the sum of the magnitudes.  24 u of the magnitudes covers the forward, and
48 u the backward's dx, whose mean adds another 14 and whose u carries the rotation's three.  A gradient of a gain adds T heads terms one after the other
at most.  What is stored in bf16 is rounded once more, by at most half its eps."""
import ctypes

import numpy as np
import pytest
import torch

from gpu_util import DEV

U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _make(B, T, Hq, Hk, D, R, dtype, layout, seed, n_pos=300):
    g = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g)
    dt = DTYPES[dtype]
    if layout == "dense":
        q, k = rn(B, T, Hq, D).to(dt).to(DEV), rn(B, T, Hk, D).to(dt).to(DEV)
    elif layout == "fused":
        x = rn(B, T, Hq + 2 * Hk, D).to(dt).to(DEV)
        q, k = x[:, :, :Hq], x[:, :, Hq:Hq + Hk]
    else:   # rows of an odd number of elements: nothing is aligned to more than an element
        ld = (Hq + Hk) * D + 3
        x = rn(B, T, ld).to(dt).to(DEV)
        q, k = x[..., 1:1 + Hq * D].unflatten(-1, (Hq, D)), x[..., 2 + Hq * D:2 + (Hq + Hk) * D].unflatten(-1, (Hk, D))
    gq, gk = (1 + 0.3 * rn(D)).to(DEV), (1 + 0.3 * rn(D)).to(DEV)
    cos = sin = pos = None
    if R:
        a = torch.arange(n_pos, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
        cos, sin = a.cos().float().to(DEV), a.sin().float().to(DEV)
        pos = torch.randint(0, n_pos, (B, T), generator=g, dtype=torch.int32).to(DEV)
    dyq, dyk = rn(B, T, Hq, D).to(dt).to(DEV), rn(B, T, Hk, D).to(dt).to(DEV)
    return q, k, gq, gk, cos, sin, pos, dyq, dyk


def _pairs(R, inter):
    j = torch.arange(R // 2)
    return (2 * j, 2 * j + 1) if inter else (j, j + R // 2)


def _turn(x, cos, sin, pos, inter, back=False, magnitude=False):
    """Rotation in 64 bits; with `magnitude` the sum of the terms' magnitudes in place of their difference."""
    if cos is None:
        return x.abs() if magnitude else x
    c, s = (t.double().cpu()[pos.long().cpu()][:, :, None] for t in (cos, sin))
    a, b = _pairs(2 * cos.shape[1], inter)
    s = -s if back else s
    out = x.clone()
    if magnitude:
        x, c, s = x.abs(), c.abs(), s.abs()
        out = out.abs()
        out[..., a], out[..., b] = x[..., a] * c + x[..., b] * s, x[..., b] * c + x[..., a] * s
    else:
        out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return out


SHAPES = [(1, 1, 1, 1, 8, 8), (2, 3, 1, 0, 16, 0), (2, 5, 3, 1, 24, 16), (3, 7, 4, 2, 64, 64), (1, 33, 12, 4, 80, 32), (2, 9, 32, 8, 128, 128), (2, 17, 5, 5, 136, 72),
          (1, 4, 2, 1, 256, 64), (1, 3, 1, 2, 512, 512), (70, 1, 0, 3, 32, 24), (1, 130, 1, 1, 96, 96)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("layout", ["dense", "fused", "odd"])
@pytest.mark.parametrize("B,T,Hq,Hk,D,R", SHAPES)
def test_forward_and_backward(dp, B, T, Hq, Hk, D, R, layout, inter, dtype):
    q, k, gq, gk, cos, sin, pos, dyq, dyk = _make(B, T, Hq, Hk, D, R, dtype, layout, B + T + D)
    eps, half = 1e-5, torch.finfo(DTYPES[dtype]).eps / 2
    yq, yk = torch.empty_like(dyq), torch.empty_like(dyk)
    dp.qk_norm(q, k, gq, gk, cos, sin, yq, yk, positions=pos, interleaved=inter, eps=eps)
    dxq, dxk = (torch.empty(t.untyped_storage().size() // t.element_size(), dtype=t.dtype, device=DEV).as_strided(t.shape, t.stride(), t.storage_offset()) for t in (q, k))
    grads = torch.empty(B, 2, D, device=DEV)
    dp.qk_norm_grads(q, k, gq, gk, cos, sin, dyq, dyk, grads, dxq, dxk, positions=pos, interleaved=inter, eps=eps)
    only = torch.empty_like(grads)
    dp.qk_norm_grads(q, k, gq, gk, cos, sin, dyq, dyk, only, positions=pos, interleaved=inter, eps=eps)
    dp.sync()
    assert torch.equal(only, grads)
    for row, (x, g, y, dy, dx) in enumerate(((q, gq, yq, dyq, dxq), (k, gk, yk, dyk, dxk))):
        x, g, dy = x.double().cpu(), g.double().cpu(), dy.double().cpu()
        H = x.shape[2]
        r = (x.pow(2).mean(-1, keepdim=True) + eps).rsqrt()
        z = x * r * g
        ref, most = _turn(z, cos, sin, pos, inter), _turn(z, cos, sin, pos, inter, magnitude=True)
        assert torch.all((y.double().cpu() - ref).abs() <= 24 * U * most * (1 + half) + half * ref.abs())
        u, um = _turn(dy, cos, sin, pos, inter, back=True), _turn(dy, cos, sin, pos, inter, back=True, magnitude=True)
        xh = x * r
        ref, most = (u * xh).sum((1, 2)), (um * xh.abs()).sum((1, 2))
        assert torch.all((grads[:, row].double().cpu() - ref).abs() <= (T * H + 40) * U * most)
        ref = r * (g * u - xh * (g * u * xh).mean(-1, keepdim=True))
        most = r * (g.abs() * um + xh.abs() * (g.abs() * um * xh.abs()).mean(-1, keepdim=True))
        assert torch.all((dx.double().cpu() - ref).abs() <= 48 * U * most * (1 + half) + half * ref.abs())


@pytest.mark.gpu
def test_gradients_are_those_of_the_forward(dp):
    """Differences of the forward in fp32 along random directions: the step of 2^-6 leaves an error of its square, the roundings of the forward
    one of 24 u over the step."""
    B, T, Hq, Hk, D, R = 2, 6, 3, 2, 48, 32
    q, k, gq, gk, cos, sin, pos, dyq, dyk = _make(B, T, Hq, Hk, D, R, "f32", "dense", 5)
    grads, dq, dk = torch.empty(B, 2, D, device=DEV), torch.empty_like(q), torch.empty_like(k)
    dp.qk_norm_grads(q, k, gq, gk, cos, sin, dyq, dyk, grads, dq, dk, positions=pos)
    vq, vk, wq, wk = (torch.randn_like(t) for t in (q, k, gq, gk))
    h = 2.0 ** -6
    ends = []
    for s in (h, -h):
        yq, yk = torch.empty_like(q), torch.empty_like(k)
        dp.qk_norm(q + s * vq, k + s * vk, gq + s * wq, gk + s * wk, cos, sin, yq, yk, positions=pos)
        ends.append((yq.double() * dyq.double()).sum() + (yk.double() * dyk.double()).sum())
    dp.sync()
    got = ((dq * vq).double().sum() + (dk * vk).double().sum() + (grads[:, 0].sum(0) * wq).double().sum() + (grads[:, 1].sum(0) * wk).double().sum()).item()
    diff = ((ends[0] - ends[1]) / (2 * h)).item()
    size = sum((t.double() ** 2).sum().item() for t in (dyq, dyk)) ** 0.5 * (sum((t.double() ** 2).sum().item() for t in (vq, vk)) ** 0.5 + 20)
    assert abs(got - diff) <= (3 * h * h + 24 * U / h) * size


@pytest.mark.gpu
def test_places_of_tokens_without_positions(dp):
    q, k, gq, gk, cos, sin, _, dyq, dyk = _make(3, 20, 2, 2, 64, 64, "f32", "dense", 6)
    pos = torch.arange(20, dtype=torch.int32, device=DEV).repeat(3, 1)
    out = []
    for p in (pos, None):
        y = [torch.empty_like(q), torch.empty_like(k), torch.empty(3, 2, 64, device=DEV), torch.empty_like(q), torch.empty_like(k)]
        dp.qk_norm(q, k, gq, gk, cos, sin, *y[:2], positions=p)
        dp.qk_norm_grads(q, k, gq, gk, cos, sin, dyq, dyk, *y[2:], positions=p)
        out.append(y)
    dp.sync()
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.gpu
@pytest.mark.parametrize("where", [-1, 300, 2 ** 31 - 1, -2 ** 31])
def test_positions_outside_the_table(dp, where):
    """Reported; the token's outputs are zero, it adds nothing, and the other tokens are what they are without it."""
    import paper_2108_01624_amd as pkg

    B, T = 2, 9
    q, k, gq, gk, cos, sin, pos, dyq, dyk = _make(B, T, 3, 2, 64, 32, "f32", "fused", 7)
    good = pos.clone()
    good[1, 4] = 0
    dy0 = [t.clone() for t in (dyq, dyk)]
    for t in dy0:
        t[1, 4] = 0
    ref = [torch.empty_like(dyq), torch.empty_like(dyk), torch.empty(B, 2, 64, device=DEV)]
    dp.qk_norm(q, k, gq, gk, cos, sin, *ref[:2], positions=good)
    dp.qk_norm_grads(q, k, gq, gk, cos, sin, *dy0, ref[2], positions=good)
    dp.sync()
    for t in ref[:2]:
        t[1, 4] = 0
    pos[1, 4] = where
    got = [torch.empty_like(t) for t in ref]
    dp.qk_norm(q, k, gq, gk, cos, sin, *got[:2], positions=pos)
    with pytest.raises(pkg.DpError) as e:
        dp.sync()
    assert e.value.status == -6
    dx = [torch.ones_like(dyq), torch.ones_like(dyk)]
    q2, k2 = q.contiguous(), k.contiguous()
    dp.qk_norm_grads(q2, k2, gq, gk, cos, sin, dyq, dyk, got[2], *dx, positions=pos)
    with pytest.raises(pkg.DpError) as e:
        dp.sync()
    assert e.value.status == -6
    assert all(torch.equal(a, b) for a, b in zip(got, ref)) and not any(t[1, 4].any() for t in dx)


@pytest.mark.gpu
def test_positions_are_not_looked_at_without_a_rotation(dp):
    q, k, gq, gk, _, _, _, dyq, dyk = _make(2, 5, 3, 1, 40, 0, "bf16", "dense", 10)
    out = []
    for p in (None, torch.full((2, 5), -7, dtype=torch.int32, device=DEV)):
        y = [torch.empty_like(q), torch.empty_like(k), torch.empty(2, 2, 40, device=DEV)]
        dp.qk_norm(q, k, gq, gk, None, None, *y[:2], positions=p)
        dp.qk_norm_grads(q, k, gq, gk, None, None, dyq, dyk, y[2], positions=p)
        dp.sync()
        out.append(y)
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.gpu
def test_zero_rows_and_no_tokens(dp):
    q, k, gq, gk, cos, sin, pos, dyq, dyk = _make(2, 3, 2, 2, 32, 32, "f32", "dense", 8)
    q[1, 1] = 0
    yq, yk, dq, dk, grads = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(k), torch.empty(2, 2, 32, device=DEV)
    dp.qk_norm(q, k, gq, gk, cos, sin, yq, yk, positions=pos, eps=1e-6)
    dp.qk_norm_grads(q, k, gq, gk, cos, sin, dyq, dyk, grads, dq, dk, positions=pos, eps=1e-6)
    assert not yq[1, 1].any() and torch.isfinite(dq).all() and torch.isfinite(grads).all()
    e = lambda *s: torch.empty(*s, device=DEV)
    dp.qk_norm(e(2, 0, 2, 32), e(2, 0, 2, 32), gq, gk, cos, sin, e(2, 0, 2, 32), e(2, 0, 2, 32))
    dp.qk_norm_grads(e(2, 0, 2, 32), e(2, 0, 2, 32), gq, gk, cos, sin, e(2, 0, 2, 32), e(2, 0, 2, 32), grads)
    dp.sync()
    assert not grads.any()


@pytest.mark.gpu
def test_small_workspace_gives_the_gradients_too():
    import paper_2108_01624_amd as pkg

    q, k, gq, gk, cos, sin, pos, dyq, dyk = _make(2, 200, 2, 2, 64, 64, "f32", "dense", 9)
    out = []
    for floats in (1, 2 * 2 * 64 * 3, 1 << 20):
        with pkg.Context(workspace_bytes=4 * floats) as small:
            grads = torch.empty(2, 2, 64, device=DEV)
            small.qk_norm_grads(q, k, gq, gk, cos, sin, dyq, dyk, grads, positions=pos)
            small.sync()
            out.append(grads)
    # each within (T heads + 40) u of the magnitudes of the sum, which are below T heads times 4 standard deviations squared here
    for g in out[1:]:
        assert (g - out[0]).abs().max() <= 2 * 440 * U * 400 * 16


def test_refusals():
    """Argument checks of the library: they come before anything touches the context's stream, so a block of zeros stands in for a context."""
    import paper_2108_01624_amd as pkg

    lib = pkg.load_library()
    ctx = ctypes.create_string_buffer(1 << 14)
    keep = np.zeros(4096, dtype=np.float32)
    p = keep.ctypes.data
    far = p + 8192
    base = dict(q=p, k=p, dt=pkg.DP_F32, ldq=16, ldk=16, gq=p, gk=p, cos=p, sin=p, n_pos=4, pos=p, inter=0, B=1, T=2, Hq=1, Hk=1, D=16, R=8, eps=1e-6)
    forward = lambda yq=far, yk=far + 1024, c=ctx, **kw: lib.dp_qk_norm(c, *dict(base, **kw).values(), yq, yk)
    back = lambda dyq=p, dyk=p, g=far, dq=far, dk=far + 1024, c=ctx, **kw: lib.dp_qk_norm_grads(c, *dict(base, **kw).values(), dyq, dyk, g, dq, dk)
    for call in (forward, back):
        assert call(c=None) == -1
        assert call(B=0) == 0
        for kw in (dict(D=12), dict(D=0), dict(D=520), dict(R=4), dict(R=24), dict(R=-8), dict(Hq=-1), dict(Hk=-1), dict(B=-1), dict(T=-1), dict(ldq=15), dict(ldk=15),
                   dict(Hq=2), dict(n_pos=-1), dict(B=1 << 20, T=1 << 20), dict(Hq=1 << 20, Hk=1)):
            assert call(**kw) == -2, kw
        for kw in (dict(q=None), dict(k=None), dict(gq=None), dict(gk=None), dict(cos=None), dict(sin=None)):
            assert call(**kw) == -1, kw
        for kw in (dict(q=p + 2), dict(k=p + 1, dt=pkg.DP_BF16), dict(gq=p + 2), dict(cos=p + 2), dict(pos=p + 2)):
            assert call(**kw) == -4, kw
        assert call(dt=3) == -3 and call(eps=0.0) == -5 and call(eps=-1.0) == -5 and call(eps=float("inf")) == -5 and call(eps=float("nan")) == -5
        assert call(eps=1e-39) == -5 and call(n_pos=0) == -2 and call(n_pos=0, B=0) == 0
    assert forward(Hq=0, Hk=0, q=None, k=None) == 0
    assert forward(yq=None) == -1 and forward(yk=None) == -1 and forward(yq=far + 2) == -4 and forward(yq=p) == -5 and forward(yk=p + 64) == -5
    assert back(dyq=None) == -1 and back(dyk=p + 2) == -4 and back(g=None) == -1 and back(dq=None) == -1 and back(dk=p) == -5 and back(dq=far + 1) == -4


def test_refusals_of_tensors():
    import paper_2108_01624_amd as pkg

    if torch.cuda.is_available():
        pytest.skip("on the CPU, where no call could touch memory")
    pkg.load_library()
    ctx = ctypes.addressof(ctypes.create_string_buffer(1 << 14))
    z = torch.zeros
    good = dict(q=z(2, 3, 2, 16), k=z(2, 3, 1, 16), gq=z(16), gk=z(16), cos=z(9, 4), sin=z(9, 4), dyq=z(2, 3, 2, 16), dyk=z(2, 3, 1, 16))
    bad = [dict(k=z(2, 4, 1, 16)), dict(k=z(2, 3, 1, 16).bfloat16()), dict(gq=z(15)), dict(gk=z(32)[::2]), dict(gk=z(16).double()), dict(cos=None), dict(cos=z(9, 8)),
           dict(sin=z(4, 9).t()), dict(dyq=z(2, 3, 16, 2).transpose(2, 3)), dict(dyk=z(2, 3, 2, 16)), dict(q=z(2, 2, 3, 16).transpose(1, 2)), dict(q=z(2, 3, 2, 32)[..., ::2]),
           dict(q=z(3, 2, 2, 16).transpose(0, 1)),
           dict(positions=z(3, 2, dtype=torch.int32)), dict(positions=z(2, 3))]
    for change in bad:
        a = dict(good, **change)
        pos = a.pop("positions", None)
        with pytest.raises((ValueError, TypeError)):
            pkg.dp_qk_norm(ctx, *list(a.values())[:6], a["dyq"], a["dyk"], positions=pos)
        with pytest.raises((ValueError, TypeError)):
            pkg.dp_qk_norm_grads(ctx, *a.values(), z(2, 2, 16), positions=pos)
    for grads, dq, dk in ((z(2, 2, 15), None, None), (z(2, 2, 16).double(), None, None), (z(2, 2, 16), z(2, 3, 2, 16), None), (z(2, 2, 16), z(2, 3, 4, 16)[:, :, :2], z(2, 3, 1, 16))):
        with pytest.raises((ValueError, TypeError)):
            pkg.dp_qk_norm_grads(ctx, *good.values(), grads, dq, dk)


def test_refusals_of_outputs_that_overlap():
    """Outputs over what is read, or over each other: refused before anything is launched.  What is allowed goes on to its launch, which fails for want
    of a GPU (-8)."""
    import paper_2108_01624_amd as pkg

    if torch.cuda.is_available():
        pytest.skip("on the CPU, where no call could touch memory")
    lib = pkg.load_library()
    ctx = ctypes.create_string_buffer(1 << 14)
    keep = np.zeros(1 << 14, dtype=np.float32)
    at = lambda k: keep.ctypes.data + 4 * k
    # two examples of three tokens, two query heads and one key head of 16 numbers, next to each other in rows of 60; what is read lies below 1,000
    B, T, Hq, Hk, D, R, ld = 2, 3, 2, 1, 16, 8, 60
    base = dict(q=at(0), k=at(32), dt=pkg.DP_F32, ldq=ld, ldk=ld, gq=at(400), gk=at(416), cos=at(432), sin=at(448), n_pos=4, pos=at(464), inter=0, B=B, T=T, Hq=Hq, Hk=Hk, D=D,
                R=R, eps=1e-6)
    nq, nk = B * T * Hq * D, B * T * Hk * D   # 192, 96
    forward = lambda yq=at(1000), yk=at(1300), **kw: lib.dp_qk_norm(ctx, *dict(base, **kw).values(), yq, yk)
    back = lambda g=at(3000), dq=at(2000), dk=at(2032), dyq=at(500), dyk=at(700), **kw: lib.dp_qk_norm_grads(ctx, *dict(base, **kw).values(), dyq, dyk, g, dq, dk)
    assert forward() == -8 and back() == -8
    # each other
    assert forward(yk=at(1000 + nq)) == -8 and forward(yk=at(1000 + nq - 1)) == -5 and forward(yk=at(1000)) == -5
    assert forward(yk=at(1000 - nk)) == -8 and forward(yk=at(1000 - nk + 1)) == -5
    # the columns that are free of dq are 32 to 59, of which dk takes 16
    for k, st in ((31, -5), (32, -8), (44, -8), (45, -5), (59, -5), (60 + 31, -5), (60 + 32, -8), (-16, -8), (-28, -8), (-29, -5), (-15, -5), (5 * 60 + 32, -8)):
        assert back(dk=at(2000 + k)) == st, k
    assert back(dk=at(2032), ldk=61) == -5   # other rows
    assert back(dq=None, dk=None) == -8
    # gains, angles, positions; the last number of one, the first of the other
    for name, n in (("gq", 16), ("gk", 16), ("cos", 16), ("sin", 16), ("pos", 6)):
        for call, out, last in ((forward, "yq", 1000 + nq - 1), (forward, "yk", 1300 + nk - 1), (back, "dq", 2000 + 5 * ld + 31), (back, "dk", 2032 + 5 * ld + 15),
                                (back, "g", 3000 + B * 2 * D - 1)):
            first = {"yq": 1000, "yk": 1300, "dq": 2000, "dk": 2032, "g": 3000}[out]
            assert call(**{name: at(last)}) == -5 and call(**{name: at(first - n + 1)}) == -5, (name, out)
            if out != "dq":
                assert call(**{name: at(last + 1)}) == -8, (name, out)
    # without a rotation nothing is read of the angles and positions
    assert forward(R=0, cos=at(1000), sin=at(1000), pos=at(1000)) == -8 and back(R=0, cos=at(2000), sin=at(3000), pos=at(3000)) == -8
    # grads over queries, keys, their gradients and the outputs
    for g in (0, 31, 5 * ld + 47, 500, 500 + nq - 1, 700, 700 + nk - 1, 2000, 2000 + 5 * ld + 31):
        assert back(g=at(g)) == -5, g
    assert back(g=at(500 + nq - 1), dq=None, dk=None) == -5 and back(g=at(2000), dq=None, dk=None) == -8
    # sides without heads have no places
    assert forward(Hk=0, k=None, gk=None, yk=None) == -8 and forward(Hk=0, yk=at(1000)) == -8 and back(Hq=0, dq=at(2032), dyq=at(3000), dk=at(2000)) == -8


def test_examples_of_more_than_a_billion_tokens_are_not_refused():
    """Without room in the workspace an example is one workgroup's: its launch is tried, and fails for want of a GPU (-8)."""
    import paper_2108_01624_amd as pkg

    if torch.cuda.is_available():
        pytest.skip("on the CPU, where no call could touch memory")
    lib = pkg.load_library()
    ctx = ctypes.create_string_buffer(1 << 14)
    at = lambda k: k << 44
    for T in (1 << 30, (1 << 30) + 1, (1 << 31) - 5000, (1 << 31) - 4097):
        args = (at(1), None, pkg.DP_BF16, 8, 8, at(2), None, None, None, 0, None, 0, 1, T, 1, 0, 8, 0, 1e-6)
        assert lib.dp_qk_norm(ctx, *args, at(3), None) == -8, T
        assert lib.dp_qk_norm_grads(ctx, *args, at(4), None, at(5), at(6), None) == -8, T


def test_sizes_beyond_32_bits_are_refused():
    """... and not cut down to what is left of them."""
    import paper_2108_01624_amd as pkg

    if torch.cuda.is_available():
        pytest.skip("on the CPU, where no call could touch memory")
    pkg.load_library()
    block = ctypes.create_string_buffer(1 << 14)
    ctx = object.__new__(pkg.Context)
    ctx.handle = ctypes.addressof(block)
    long, z = (1 << 32) + 1, torch.zeros
    g, x = z(16), z(2, 3, 1, 16)
    for call in (lambda: ctx.qk_norm(z(0, long, 1, 16), z(0, long, 1, 16), g, g, None, None, z(0, long, 1, 16), z(0, long, 1, 16)),
                 lambda: ctx.qk_norm_grads(z(long, 0, 1, 16), z(long, 0, 1, 16), g, g, None, None, z(long, 0, 1, 16), z(long, 0, 1, 16),
                                           z(1).expand(long, 2, 16)),
                 lambda: ctx.qk_norm(x, x, g, g, z(long, 0), z(long, 0), z(2, 3, 1, 16), z(2, 3, 1, 16))):
        with pytest.raises(pkg.DpError) as e:
            call()
        assert e.value.status == -2
    ctx.handle = None
