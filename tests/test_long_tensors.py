"""Held gradients, bias and query/key tensors of more than 2^32 bytes and elements: what lies behind these offsets is compared with the same call on a
copy of it alone (bit for bit where the order of the additions is the same), or with a sum in 64 bits."""
import pytest
import torch

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


def _pattern(n, dtype, seed):
    """n numbers: a drawn million, repeated."""
    base = torch.randn(1 << 20, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)
    return base.repeat((n + base.numel() - 1) // base.numel())[:n]


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def test_held_gradient_of_one_unit(dp):
    n = (1 << 32) + (1 << 31) + 12_345   # three entries of a table
    x = _pattern(n, torch.bfloat16, 1)
    sq, S = torch.zeros(1, device=DEV), torch.zeros(n, device=DEV)
    dp.sqnorms_grads([x], sq)
    ref = sum((c.double() ** 2).sum().item() for c in x.split(1 << 28))
    # 9 + 9 additions in a workgroup's piece, 394,000 / 1,024 / 4 + 3 in a lane of their sum, 10 over its workgroup
    assert abs(sq.item() - ref) <= 160 * 2.0 ** -24 * ref
    C = 0.5 * ref ** 0.5
    dp.clip_accumulate_grads([x], C, sq, [S])
    dp.clip_grads([x], C, sq, [x])
    dp.sync()
    for a in (0, (1 << 31) - 5000, (1 << 32) - 5000, n - 10_000):
        want = _pattern(1 << 20, torch.bfloat16, 1)[torch.arange(a, min(a + 10_000, n), device=DEV) % (1 << 20)].double() * 0.5
        for got, eps in ((S, 0.0), (x, 2.0 ** -8)):
            got = got[a:a + 10_000].double()
            assert torch.all((got - want).abs() <= (100 * 2.0 ** -24 + eps) * want.abs())


def test_held_gradients_of_several_units(dp):
    B, n = 3, 1_500_000_007
    x = _pattern(B * n, torch.bfloat16, 2).view(B, n)
    sq, one = torch.zeros(B, device=DEV), torch.zeros(1, device=DEV)
    dp.sqnorms_grads([x], sq)
    dp.sqnorms_grads([x[2]], one)
    assert abs(sq[2].item() - one.item()) <= 200 * 2.0 ** -24 * one.item()
    S = torch.zeros(n, device=DEV)
    dp.clip_accumulate_grads([x], 1.0, sq, [S])
    dp.sync()
    c = torch.clamp(1.0 / sq.double().sqrt(), max=1.0)
    for a in (0, n - 10_001):
        part = x[:, a:a + 10_001].double() * c[:, None]
        assert torch.all((S[a:a + 10_001].double() - part.sum(0)).abs() <= 16 * 2.0 ** -24 * part.abs().sum(0))


def test_bias_and_its_gradient(dp):
    H, T, starts = 17, 16384, [0, 1, 2, 3, 5, 8, 13, 200]
    table = torch.randn(16, H, device=DEV)
    bias, last = torch.empty(H, T, T, dtype=torch.bfloat16, device=DEV), torch.empty(1, T, T, dtype=torch.bfloat16, device=DEV)
    dp.relative_bias(table, starts, True, bias)
    dp.relative_bias(table[:, -1:].contiguous(), starts, True, last)
    assert torch.equal(bias[-1:], last)
    del bias, last
    B, T = 70, 2001
    dS = _pattern(B * 16 * T * T, torch.bfloat16, 3).view(B, 16, T, T)
    grads, one = torch.empty(B, 16, 16, device=DEV), torch.empty(1, 16, 16, device=DEV)
    for causal in (False, True):
        dp.relative_bias_grads([dS], starts, True, grads, causal=causal)
        dp.relative_bias_grads([dS[-1:].clone()], starts, True, one, causal=causal)
        dp.sync()
        size = dS[-1].float().abs().sum((1, 2))   # of a bucket's terms at most; T + T / 64 + 40 additions either way
        assert torch.all((grads[-1] - one[0]).abs() <= 2 * (T + T / 64 + 40) * 2.0 ** -24 * size)


def test_queries_and_keys(dp):
    B, T, H, D = 72, 4001, 120, 128
    x = _pattern(B * T * H * D, torch.bfloat16, 4).view(B, T, H, D)
    q, k = x[:, :, :100], x[:, :, 100:]
    g = torch.randn(2, D, device=DEV)
    a = torch.rand(T, D // 2, device=DEV)
    dyq, dyk = _pattern(q.numel(), torch.bfloat16, 5).view(q.shape), _pattern(k.numel(), torch.bfloat16, 6).view(k.shape)
    yq, yk, dx, grads = torch.empty_like(dyq), torch.empty_like(dyk), torch.empty_like(x), torch.empty(B, 2, D, device=DEV)
    dp.qk_norm(q, k, g[0], g[1], a.cos(), a.sin(), yq, yk)
    dp.qk_norm_grads(q, k, g[0], g[1], a.cos(), a.sin(), dyq, dyk, grads, dx[:, :, :100], dx[:, :, 100:])
    dp.sync()
    one = x[-1:].clone()
    out = [torch.empty_like(t[-1:]) for t in (yq, yk)]
    d1, g1 = torch.empty_like(one), torch.empty(1, 2, D, device=DEV)
    dp.qk_norm(one[:, :, :100], one[:, :, 100:], g[0], g[1], a.cos(), a.sin(), *out)
    dp.qk_norm_grads(one[:, :, :100], one[:, :, 100:], g[0], g[1], a.cos(), a.sin(), dyq[-1:].clone(), dyk[-1:].clone(), g1, d1[:, :, :100], d1[:, :, 100:])
    dp.sync()
    assert torch.equal(out[0], yq[-1:]) and torch.equal(out[1], yk[-1:]) and torch.equal(d1, dx[-1:])
    size = torch.stack([dyq[-1].float().abs().sum((0, 1)), dyk[-1].float().abs().sum((0, 1))]) * 8   # a normalised number is below 8 here
    assert torch.all((grads[-1] - g1[0]).abs() <= 2 * (T + 100) * 2.0 ** -24 * size)


def test_queries_of_an_example_of_two_billion_tokens(dp):
    """Nearly 2^31 tokens of one example: the first and last ones, which alone have a gradient, against the same calls on a copy of them, and the gain's
    gradient against its sum in 64 bits (2,000 terms, a rounding each for u, xhat, their product and the sum)."""
    T, D, n = (1 << 31) - 5000, 8, 1000
    q = _pattern(T * D, torch.bfloat16, 7).view(1, T, 1, D)
    none = torch.empty(1, T, 0, D, dtype=torch.bfloat16, device=DEV)
    g = torch.linspace(0.5, 2, D, device=DEV)
    y, dy, grads = torch.empty_like(q), torch.zeros_like(q), torch.empty(1, 2, D, device=DEV)
    dy[:, :n] = q[:, 5 * n:6 * n]
    dy[:, -n:] = q[:, 7 * n:8 * n]
    ends = lambda t: torch.cat([t[:, :n], t[:, -n:]], 1)
    x, d = ends(q), ends(dy)
    few, y1, dx1, g1 = none[:, :2 * n], torch.empty_like(x), torch.empty_like(x), torch.empty_like(grads)
    dp.qk_norm(q, none, g, g, None, None, y, none)
    dp.qk_norm(x, few, g, g, None, None, y1, few)
    dp.sync()
    assert torch.equal(ends(y), y1)
    dp.qk_norm_grads(q, none, g, g, None, None, dy, none, grads, y, none)
    dp.qk_norm_grads(x, few, g, g, None, None, d, few, g1, dx1, few)
    dp.sync()
    assert torch.equal(ends(y), dx1) and not y[:, n:n + 5000].any() and not y[:, -2 * n:-n].any()
    x, d = x.double().flatten(0, 2), d.double().flatten(0, 2)
    terms = d * x * (x.pow(2).mean(-1, keepdim=True) + 1e-6).rsqrt()
    assert torch.all((grads[0, 0].double() - terms.sum(0)).abs() <= (2 * n + 40) * 2.0 ** -24 * terms.abs().sum(0)) and not grads[0, 1].any()
