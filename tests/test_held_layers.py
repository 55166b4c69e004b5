"""Layers whose per-example gradients exist as tensors, through the step driver: adapters that the caller differentiates, a relative position bias
shared by two attention layers and norms of queries and keys, next to dense, LayerNorm and embedding layers.  One whole step against a computation in
64 bits, its replay from a HIP graph, two streams, and the calls that the driver and the extension make."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.append(ROOT)   # (behind the package on the stub, where there is one)

import dp_synth as syn  # noqa: E402
from oracle import dp_oracle as orc  # noqa: E402

DEV = "cuda:0"
STARTS = [0, 1, 2, 3, 4, 6, 9, 14]


class Spec:
    def __init__(self, *shapes):
        self.shapes = shapes

    def tensors(self):
        return [(str(k), s) for k, s in enumerate(self.shapes)]


def manifest(d, H, D, V):
    return [Spec((V, d)), Spec((2 * len(STARTS), H)), Spec((d, d), (d,)), Spec((D,), (D,)), Spec((d,), (d,)), Spec((d, 3), (3, d), (5,)), Spec((d, d), (d,))]


def micro_batch(B, T, d, H, D, V, seed, device=DEV, dtype=torch.bfloat16):
    """Bias and scores of two layers, one padded length per example, rotated heads of a fused projection, adapters in fp32 and one in bf16."""
    g = torch.Generator().manual_seed(seed)
    rn = lambda *s, dt=dtype, k=1.0: (torch.randn(*s, generator=g) * k).to(dt).to(device)
    scale = torch.logspace(-1, 1, B)[torch.randperm(B, generator=g)].to(device)
    sc = lambda t: (t * scale.view((-1,) + (1,) * (t.dim() - 1))).to(t.dtype)
    qkv = rn(B, T, 3 * H, D)
    a = torch.arange(T, dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    ids = torch.randint(0, V, (B, T), generator=g, dtype=torch.int32).to(device)
    lengths = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32).to(device)
    return [
        dict(kind="embedding", ids=ids, G=sc(rn(B, T, d, k=0.1)), V=V, distinct=False),
        dict(kind="relative_bias", dS=[sc(rn(B, H, T, T, k=0.05)) for _ in range(2)], starts=STARTS, bidirectional=True, lengths=lengths),
        dict(kind="dense", A=rn(B, T, d), G=sc(rn(B, T, d, k=0.02)), has_bias=True),
        dict(kind="qk_norm", q=qkv[:, :, :H], k=qkv[:, :, H:2 * H], gain_q=rn(D, dt=torch.float32), gain_k=rn(D, dt=torch.float32), cos=a.cos().float().to(device),
             sin=a.sin().float().to(device), dyq=sc(rn(B, T, H, D, k=0.1)), dyk=sc(rn(B, T, H, D, k=0.1)), eps=1e-5),
        dict(kind="layernorm", X=rn(B, T, d), G=sc(rn(B, T, d, k=0.05))),
        dict(kind="grads", grads=[sc(rn(B, d, 3, dt=torch.float32, k=0.3)), sc(rn(B, 3, d, dt=torch.float32, k=0.3)), sc(rn(B, 5, k=0.5))]),
        dict(kind="dense", A=rn(B, T, d), G=sc(rn(B, T, d, k=0.02)), has_bias=True),
    ]


def example_gradients(layers):
    """Per layer and tensor, [B, ...] in 64 bits: written out from the definitions."""
    out = []
    for l in layers:
        f = lambda k: l[k].double().cpu()
        if l["kind"] == "dense":
            out.append([f("A").transpose(1, 2) @ f("G"), f("G").sum(1)])
        elif l["kind"] == "layernorm":
            out.append([(f("X") * f("G")).sum(1), f("G").sum(1)])
        elif l["kind"] == "embedding":
            e = torch.zeros(l["ids"].shape[0], l["V"], l["G"].shape[2], dtype=torch.float64)
            for i, row in enumerate(l["ids"].cpu().long()):
                e[i].index_add_(0, row, f("G")[i])
            out.append([e])
        elif l["kind"] == "grads":
            out.append([t.double().cpu() for t in l["grads"]])
        elif l["kind"] == "relative_bias":
            B, H, T, _ = l["dS"][0].shape
            rel = torch.arange(T)[None, :] - torch.arange(T)[:, None]
            b = (rel.abs()[..., None] >= torch.tensor(STARTS)).sum(-1) - 1 + len(STARTS) * (rel > 0)
            e = torch.zeros(B, H, 2 * len(STARTS), dtype=torch.float64)
            for x in l["dS"]:
                x = x.double().cpu()
                for i, n in enumerate(l["lengths"].tolist()):
                    e[i].index_add_(1, b[:n, :n].flatten(), x[i, :, :n, :n].reshape(H, -1))
            out.append([e.transpose(1, 2)])
        else:
            T, D = l["q"].shape[1], l["q"].shape[3]
            c, s = f("cos")[None, :, None], f("sin")[None, :, None]
            both = []
            for n in "qk":
                x, dy = f(n), f("dy" + n)
                y1, y2 = dy[..., :D // 2], dy[..., D // 2:]
                u = torch.cat([y1 * c + y2 * s, y2 * c - y1 * s], -1)
                both.append((u * x * (x.pow(2).mean(-1, keepdim=True) + l["eps"]).rsqrt()).sum((1, 2)))
            out.append(both)
    return out


SIZES = dict(B=9, T=24, d=32, H=3, D=16, V=50)


@pytest.mark.gpu
@pytest.mark.parametrize("batch_dense", [True, False])
def test_step_over_held_and_other_layers(dp, batch_dense):
    """Norms, sums and update of two micro-batches.  Tolerances: the framework's own for bf16 layers (their sums may pass through bf16 once), 2e-2 of
    a norm and of a tensor's sum; the held layers are fp32 sums of fewer than 2^10 terms, 2^-14 of the sum of the magnitudes, on top of the norms' part."""
    import paper_2108_01624_amd as pkg

    C, s = 1.0, SIZES
    run = pkg.StepRunner(dp, manifest(s["d"], s["H"], s["D"], s["V"]), s["B"], device=DEV)
    ref = None
    for m, B in enumerate((s["B"], s["B"] - 2)):
        layers = micro_batch(**dict(s, B=B), seed=m)
        grads = example_gradients(layers)
        n = sum((t.flatten(1) ** 2).sum(1) for per in grads for t in per)
        got = run.pass1(layers, batch_dense=batch_dense)
        assert got.shape == (B,)
        np.testing.assert_allclose(got.cpu().double().numpy(), n.numpy(), rtol=2e-2)
        run.pass2(layers, C, batch_dense=batch_dense)
        c = torch.clamp(C / n.sqrt(), max=1.0)
        assert (c < 1).any() and (c == 1).any()
        # the clip factors that pass 2 used are those of the norms it was given
        c = torch.clamp(C / got.cpu().double().sqrt(), max=1.0)
        part = [[(torch.tensordot(c, t, 1), torch.tensordot(c, t.abs(), 1)) for t in per] for per in grads]
        ref = part if ref is None else [[(a + x, b + y) for (a, b), (x, y) in zip(p, q)] for p, q in zip(ref, part)]
    dp.sync()
    for k, per in enumerate(ref):
        for j, (sums, most) in enumerate(per):
            got = run.view(run.S, k, j).cpu().double()
            held = layers[k]["kind"] in ("grads", "relative_bias", "qk_norm")
            if held:
                assert torch.all((got - sums).abs() <= 2.0 ** -14 * most), (k, j)
            assert (got - sums).norm() <= (1e-4 if held else 2e-2) * most.norm(), (k, j)
    theta0, S = syn.normal_f32((run.P,), 0.02, 3), run.S.cpu().numpy().copy()
    run.theta.copy_(torch.from_numpy(theta0))
    kw = dict(sigma=0.5, C=C, seed=11, step=1, batch_size=16, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-11, weight_decay=0.1)
    run.update(**kw)
    dp.sync()
    th, m_, v_, _ = orc.noise_adamw(theta0, np.zeros_like(theta0), np.zeros_like(theta0), S, elem_offset=0, **kw)
    np.testing.assert_allclose(run.m.cpu().numpy(), m_, rtol=1e-4, atol=1e-6 * np.abs(m_).max())
    assert not run.S.any()


@pytest.mark.gpu
def test_replay_from_a_graph_and_two_streams():
    """A captured pass 1 and pass 2 with held layers, and the backward of queries and keys with its outputs, replayed with other inputs between eager
    work, bit for bit the eager calls; a second context on another stream at the same time."""
    import paper_2108_01624_amd as pkg

    s, C = SIZES, 1.0
    side, other = torch.cuda.Stream(device=DEV), torch.cuda.Stream(device=DEV)
    inputs = [micro_batch(**s, seed=20 + k) for k in range(3)]

    def tensors(layers):
        return [t for l in layers for v in l.values() for t in (v if isinstance(v, list) else [v]) if torch.is_tensor(t)]

    def start(stream):
        with torch.cuda.stream(stream):
            ctx = pkg.Context()
            run = pkg.StepRunner(ctx, manifest(s["d"], s["H"], s["D"], s["V"]), s["B"], device=DEV)
            layers = micro_batch(**s, seed=1)
            layers[3]["dq"], layers[3]["dk"] = torch.empty_strided(layers[3]["q"].shape, layers[3]["q"].stride(), dtype=torch.bfloat16, device=DEV), \
                torch.empty_strided(layers[3]["k"].shape, layers[3]["k"].stride(), dtype=torch.bfloat16, device=DEV)
        return ctx, run, layers

    def load(layers, k):
        for a, b in zip(tensors([{q: v for q, v in l.items() if q not in ("dq", "dk")} for l in layers]), tensors(inputs[k])):
            a.copy_(b)

    def result(run, layers):
        return [t.cpu().clone() for t in (run.sqnorms, run.S, layers[3]["dq"], layers[3]["dk"])]

    ctx, run, layers = start(side)
    ctx2, run2, layers2 = start(other)
    torch.cuda.synchronize()
    refs = []
    with torch.cuda.stream(side):
        for k in range(3):
            load(layers, k)
            run.S.zero_()
            run.pass1(layers)
            run.pass2(layers, C)
            ctx.sync()
            refs.append(result(run, layers))
        graph = torch.cuda.CUDAGraph()
        run.S.zero_()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            run.pass1(layers)
            run.pass2(layers, C)
    for k in (2, 0, 1, 1):
        with torch.cuda.stream(other):
            load(layers2, (k + 1) % 3)
            run2.S.zero_()
        with torch.cuda.stream(side):
            load(layers, k)
            run.S.zero_()
        torch.cuda.synchronize()
        graph.replay()   # (on the current stream)
        with torch.cuda.stream(other):
            run2.pass1(layers2)
            run2.pass2(layers2, C)
        torch.cuda.synchronize()
        ctx.sync()
        ctx2.sync()
        assert all(torch.equal(a, b) for a, b in zip(result(run, layers), refs[k]))
        assert all(torch.equal(a, b) for a, b in zip(result(run2, layers2), refs[(k + 1) % 3]))
    del graph
    ctx.close()
    ctx2.close()


@pytest.mark.gpu
def test_calls_through_the_extension_are_those_of_the_functions(dp):
    """A context's methods against the functions of the same names: the same bits, and the same refusals."""
    import paper_2108_01624_amd as pkg

    s = SIZES
    l = micro_batch(**s, seed=5)
    bias, qk, held = l[1], l[3], l[5]["grads"]
    B = s["B"]
    new = lambda *shape: torch.zeros(*shape, device=DEV)

    def both(name, make, *a, **k):
        outs = []
        for call in (getattr(dp, name), lambda *a, **k: getattr(pkg, "dp_" + name)(dp.handle, *a, **k)):
            out = make()
            call(*[x(out) if callable(x) else x for x in a], **k)
            outs.append(out)
        dp.sync()
        for x, y in zip(*outs):
            assert torch.equal(x, y), name

    both("sqnorms_grads", lambda: [new(B)], held[:2], lambda o: o[0])
    sq = new(B)
    dp.sqnorms_grads(held[:2], sq)
    both("clip_accumulate_grads", lambda: [new(s["d"], 3), new(3, s["d"])], held[:2], 1.0, sq, lambda o: list(o))
    both("clip_grads", lambda: [torch.zeros_like(t) for t in held[:2]], held[:2], 1.0, sq, lambda o: list(o))
    table = torch.randn(2 * len(STARTS), s["H"], device=DEV)
    both("relative_bias", lambda: [new(s["H"], 5, 9)], table, STARTS, True, lambda o: o[0])
    both("relative_bias_grads", lambda: [new(B, 2 * len(STARTS), s["H"])], bias["dS"], STARTS, True, lambda o: o[0], lengths=bias["lengths"])
    args = [qk[n] for n in ("q", "k", "gain_q", "gain_k", "cos", "sin")]
    both("qk_norm", lambda: [torch.zeros_like(qk["dyq"]), torch.zeros_like(qk["dyk"])], *args, lambda o: o[0], lambda o: o[1])
    both("qk_norm_grads", lambda: [new(B, 2, s["D"]), torch.zeros_like(qk["q"]), torch.zeros_like(qk["k"])], *args, qk["dyq"], qk["dyk"], lambda o: o[0])
    # refused alike, with nothing written
    host = torch.zeros(B)
    for call in (lambda: dp.sqnorms_grads([held[0].cpu()], sq), lambda: dp.sqnorms_grads(held[:2], host), lambda: dp.sqnorms_grads([held[0].transpose(1, 2)], sq),
                 lambda: dp.sqnorms_grads(held, sq), lambda: dp.clip_grads(held[:2], 1.0, sq, held[1:]), lambda: dp.clip_accumulate_grads(held[:1], 1.0, sq, [new(5)]),
                 lambda: dp.relative_bias(table, STARTS, False, new(s["H"], 5, 9)), lambda: dp.relative_bias(table, [0, 2, 1] + STARTS[3:], True, new(s["H"], 5, 9)),
                 lambda: dp.relative_bias_grads(bias["dS"], STARTS, True, new(B, 2 * len(STARTS), s["H"]), lengths=bias["lengths"].long()),
                 lambda: dp.qk_norm(*args, qk["dyq"][:, :, :2], qk["dyk"]), lambda: dp.qk_norm(*args, qk["q"], qk["k"]), lambda: dp.qk_norm(*args, qk["dyq"], qk["dyk"], eps=0.0),
                 lambda: dp.qk_norm(*args[:4], args[4].double(), args[5], qk["dyq"], qk["dyk"])):
        with pytest.raises((ValueError, TypeError, pkg.DpError)):
            call()
    dp.sync()


def held_calls():
    """(in a process on the stub of test_step_calls) the calls of a step, and its refusals."""
    from test_step_calls import _package

    pkg, context, lines = _package()
    s = dict(SIZES, B=4)
    for batch_dense in (True, False):
        run = pkg.StepRunner(context(), manifest(s["d"], s["H"], s["D"], s["V"]), 4, device="cpu")
        layers = micro_batch(**s, seed=1, device="cpu")
        try:
            run.pass2(layers, 1.0)
            raise AssertionError("pass 2 without pass 1")
        except ValueError as e:
            assert "pass1" in str(e)
        assert not lines()
        run.pass1(layers, batch_dense=batch_dense)
        names = [x.split()[0] for x in lines()]
        assert names[:5] == ["dp_zero_f32", "dp_relative_bias_grads", "dp_qk_norm_grads", "dp_sqnorms_grads", "dp_sqnorms_grads"], names
        assert sorted(names[5:]) == sorted(["dp_sqnorms_embedding"] + (["dp_sqnorms_layernorm_keep", "dp_sqnorms_dense_batched"] if batch_dense else
                                                                      ["dp_sqnorms_dense"] * 2 + ["dp_sqnorms_layernorm"])), names
        run.pass2(layers, 1.0, batch_dense=batch_dense)
        got = lines()
        names = [x.split()[0] for x in got]
        assert names[:2] == ["dp_clip_accumulate_grads"] * 2 and len(names) == (5 if batch_dense else 6), names
        # the dense sums go where the manifest puts their tensors, behind those of the held layers
        at = [run.view(run.S, k, j).data_ptr() for k in (2, 6) for j in (0, 1)]
        text = " ".join(x for x in got if "dense" in x)
        assert all(hex(p)[2:] in text for p in at), (text, [hex(p) for p in at])
        for k, change in ((5, dict(grads=layers[5]["grads"][:2])), (5, dict(grads=[t[:3] for t in layers[5]["grads"]])), (3, dict(q=layers[3]["q"][:3])),
                          (2, dict(A=layers[2]["A"][:3], G=layers[2]["G"][:3])), (1, dict(starts=STARTS[:4]))):
            wrong = [dict(l, **change) if j == k else l for j, l in enumerate(layers)]
            for call in (lambda: run.pass1(wrong, batch_dense=batch_dense), lambda: run.pass2(wrong, 1.0, batch_dense=batch_dense)):
                try:
                    call()
                except ValueError:
                    continue
                raise AssertionError(f"not refused: {change.keys()}")
            lines()
        # only held layers
        run = pkg.StepRunner(context(), [Spec((7,))], 4, device="cpu")
        run.pass1([dict(kind="grads", grads=[torch.zeros(4, 7)])])
        run.pass2([dict(kind="grads", grads=[torch.zeros(4, 7)])], 1.0)
        assert [x.split()[0] for x in lines()] == ["dp_zero_f32", "dp_sqnorms_grads", "dp_clip_accumulate_grads"]


def test_calls_of_a_step_with_held_layers(tmp_path):
    from paper_2108_01624_amd import build
    from test_step_calls import PKG, _stub_source

    if torch.cuda.is_available():
        pytest.skip("tensors of the CPU beside a stub: where there is no GPU")
    import shutil

    (tmp_path / PKG).mkdir()
    for f in os.listdir(build.PKG_DIR):
        if f.endswith(".py"):
            shutil.copy(os.path.join(build.PKG_DIR, f), tmp_path / PKG / f)
    shutil.copy(build.NATIVE_PATH, tmp_path / PKG / "_native.so")
    (tmp_path / "stub.cpp").write_text(_stub_source())
    r = subprocess.run(["g++", "-shared", "-fPIC", "-O1", "-std=c++17", "-I" + build.INCLUDE, "-Wl,-soname,libdpclip.so", str(tmp_path / "stub.cpp"),
                        "-o", str(tmp_path / PKG / "libdpclip.so")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([sys.executable, os.path.abspath(__file__), "held_calls"], capture_output=True, text=True, cwd=tmp_path, timeout=600,
                       env=dict(os.environ, PYTHONPATH=str(tmp_path)))
    assert r.returncode == 0, (r.stdout + r.stderr)[-8000:]


def kept_gradients_are_those_of_pass_1():
    """(in a process on the stub of test_step_calls) pass 2 takes the gradients that pass 1 left for these very layers, or refuses."""
    from test_step_calls import _package

    pkg, context, lines = _package()
    s = dict(SIZES, B=4)
    specs = manifest(s["d"], s["H"], s["D"], s["V"])
    run = pkg.StepRunner(context(), specs, 4, device="cpu")
    first, second = (micro_batch(**s, seed=k, device="cpu") for k in (1, 2))

    def refused(call, layers):
        lines()
        try:
            call(layers)
        except ValueError:
            assert not [x for x in lines() if "clip_accumulate" in x]
            return
        raise AssertionError("not refused")

    two = lambda layers: run.pass2(layers, 1.0)
    run.pass1(first)
    two(first)
    two(first)                                             # (again, say with another clip norm)
    two([dict(l) for l in first])                          # the same tensors in other dicts
    refused(two, second)                                   # another micro-batch of as many examples
    run.pass1(second)
    refused(two, first)
    two(second)
    buffers = {k: b.data_ptr() for k, b in run.grad_keep.items()}
    change = lambda k, **c: [dict(l, **c) if j == k else l for j, l in enumerate(second)]
    bias, qk = second[1], second[3]
    for k, c in ((1, dict(dS=bias["dS"][::-1])), (1, dict(dS=bias["dS"][:1])), (1, dict(lengths=None)), (1, dict(causal=True)), (1, dict(lengths=bias["lengths"].clone())),
                 (1, dict(starts=[0] + bias["starts"][:-1])), (3, dict(eps=1e-3)), (3, dict(interleaved=True)), (3, dict(cos=qk["sin"])), (3, dict(cos=None, sin=None)),
                 (3, dict(positions=torch.zeros(4, s["T"], dtype=torch.int32))), (3, dict(q=qk["k"])), (3, dict(dyk=qk["dyq"])),
                 (3, dict(q=qk["q"].contiguous()))):
        refused(two, change(k, **c))
    two(second)
    two(change(5, grads=[t.clone() for t in second[5]["grads"]]))   # what the caller holds is read from where it is
    # layers that are refused leave the gradients and the places of their buffers alone (a captured graph writes there)
    larger = [dict(starts=list(range(9))), dict(bidirectional=False), dict(dS=[torch.zeros(4, s["H"] + 1, s["T"], s["T"])] * 2)]
    for c in larger:
        refused(two, change(1, **c))
        two(second)
    for c in larger:
        refused(run.pass1, change(1, **c))
    run.pass1(second)
    two(second)
    assert buffers == {k: b.data_ptr() for k, b in run.grad_keep.items()}
    # after a pass 1 without such layers there is nothing to be taken
    dense = [second[2]]
    run.pass1(dense)
    refused(two, second)
    # a table of the manifest that the layer has not: refused, where it is too small as well
    for shapes in (((2 * len(STARTS), s["H"]), (5,)), ((2 * len(STARTS) * s["H"] + 1,),), ((s["H"], 2 * len(STARTS)),), ((len(STARTS), s["H"]),)):
        other = pkg.StepRunner(context(), [Spec(*shapes)], 4, device="cpu")
        refused(other.pass1, [bias])
        assert not other.grad_keep
    other = pkg.StepRunner(context(), [Spec((5,))], 4, device="cpu")
    refused(other.pass1, [dict(kind="grads", grads=[])])
    refused(other.pass1, [dict(bias, dS=[])])


def shapes_of_held_gradients():
    """(in a process on the stub of test_step_calls) gradients have the shape of the manifest's tensor, or one with axes split or joined."""
    from test_step_calls import _package

    pkg, context, lines = _package()
    run = pkg.StepRunner(context(), [Spec((6, 3), (4, 1, 5), ())], 4, device="cpu")
    z = torch.zeros
    good = ((4, 6, 3), (4, 4, 1, 5), (4,))
    for change in ((), (0, (4, 18)), (0, (4, 6, 1, 3)), (1, (4, 4, 5)), (1, (4, 20)), (1, (4, 2, 2, 5)), (0, (4, 2, 3, 3)), (2, (4, 1))):
        grads = [z(change[1] if change and change[0] == k else s) for k, s in enumerate(good)]
        run.pass1([dict(kind="grads", grads=grads)])
        run.pass2([dict(kind="grads", grads=grads)], 1.0)
        assert [x.split()[0] for x in lines()] == ["dp_zero_f32", "dp_sqnorms_grads", "dp_clip_accumulate_grads"]
    for k, shape in ((0, (4, 3, 6)), (0, (4, 2, 9)), (0, (4, 6, 2)), (0, (4, 17)), (1, (4, 5, 4)), (1, (4, 5, 1, 4)), (1, (4, 2, 10)), (0, (4, 3, 2, 3, 1, 2)), (2, (4, 2)), (2, ()), (0, ()), (0, (3, 6, 3)), (1, (5, 4, 1, 5))):
        grads = [z(shape if j == k else s) for j, s in enumerate(good)]
        for call in (run.pass1, lambda layers: run.pass2(layers, 1.0)):
            try:
                call([dict(kind="grads", grads=grads)])
            except ValueError:
                assert all(x.split()[0] == "dp_zero_f32" for x in lines())
                continue
            raise AssertionError(f"not refused: {shape}")


def flat_tensors_of_the_manifest():
    """(in a process on the stub of test_step_calls) a manifest that names the numbers of a tensor only: gradients and tables of any shape."""
    from test_step_calls import _package

    pkg, context, lines = _package()
    s = dict(SIZES, B=4)
    layers = micro_batch(**s, seed=1, device="cpu")
    layers = [layers[1], dict(kind="grads", grads=[torch.zeros(4, 2, 3, 5), torch.zeros(4, 6, 1)])]
    run = pkg.StepRunner(context(), [Spec((2 * len(STARTS) * s["H"],)), Spec((2, 15), (6,))], 4, device="cpu")
    run.pass1(layers)
    run.pass2(layers, 1.0)
    assert [x.split()[0] for x in lines()] == ["dp_zero_f32", "dp_relative_bias_grads", "dp_sqnorms_grads", "dp_clip_accumulate_grads"]
    try:
        run.pass1([layers[0], dict(kind="grads", grads=[torch.zeros(4, 2, 3, 4), torch.zeros(4, 6)])])
    except ValueError:
        return
    raise AssertionError("not refused")


def scalar_parameters():
    """(in a process on the stub of test_step_calls) a tensor of no axes, next to others."""
    from test_step_calls import _package

    pkg, context, lines = _package()
    run = pkg.StepRunner(context(), [Spec((), (3,)), Spec(())], 4, device="cpu")
    layers = [dict(kind="grads", grads=[torch.zeros(4), torch.zeros(4, 3)]), dict(kind="grads", grads=[torch.zeros(4, 1)])]
    run.pass1(layers)
    run.pass2(layers, 1.0)
    assert [x.split()[0] for x in lines()] == ["dp_zero_f32", "dp_sqnorms_grads", "dp_clip_accumulate_grads"]
    assert run.view(run.S, 0, 0).shape == () and run.view(run.theta, 0, 1).shape == (3,) and run.P == 9


def _on_the_stub(tmp_path, name):
    """Runs the function of that name, above, in a process whose package stands on the stub."""
    import shutil

    from paper_2108_01624_amd import build
    from test_step_calls import PKG, _stub_source

    (tmp_path / PKG).mkdir()
    for f in os.listdir(build.PKG_DIR):
        if f.endswith(".py"):
            shutil.copy(os.path.join(build.PKG_DIR, f), tmp_path / PKG / f)
    shutil.copy(build.NATIVE_PATH, tmp_path / PKG / "_native.so")
    (tmp_path / "stub.cpp").write_text(_stub_source())
    r = subprocess.run(["g++", "-shared", "-fPIC", "-O1", "-std=c++17", "-I" + build.INCLUDE, "-Wl,-soname,libdpclip.so", str(tmp_path / "stub.cpp"),
                        "-o", str(tmp_path / PKG / "libdpclip.so")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([sys.executable, os.path.abspath(__file__), name], capture_output=True, text=True, cwd=tmp_path, timeout=600,
                       env=dict(os.environ, PYTHONPATH=str(tmp_path)))
    assert r.returncode == 0, (r.stdout + r.stderr)[-8000:]


def test_kept_gradients_are_those_of_pass_1(tmp_path):
    if torch.cuda.is_available():
        pytest.skip("tensors of the CPU beside a stub: where there is no GPU")
    _on_the_stub(tmp_path, "kept_gradients_are_those_of_pass_1")


def test_flat_tensors_of_the_manifest(tmp_path):
    if torch.cuda.is_available():
        pytest.skip("tensors of the CPU beside a stub: where there is no GPU")
    _on_the_stub(tmp_path, "flat_tensors_of_the_manifest")


def test_scalar_parameters(tmp_path):
    if torch.cuda.is_available():
        pytest.skip("tensors of the CPU beside a stub: where there is no GPU")
    _on_the_stub(tmp_path, "scalar_parameters")


def test_shapes_of_held_gradients(tmp_path):
    if torch.cuda.is_available():
        pytest.skip("tensors of the CPU beside a stub: where there is no GPU")
    _on_the_stub(tmp_path, "shapes_of_held_gradients")


if __name__ == "__main__":
    globals()[sys.argv[1]]()
