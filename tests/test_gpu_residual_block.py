"""The operators together: a residual block of dense layers as a program learns it (norm, two dense layers, dropout, the stream's addition, and back),
and as it then serves it in 8 bits (weights brought to 8 bits once; norm into 8 bits, product, rows into 8 bits, product), on rows of the served state."""
import numpy as np
import pytest
import torch

import block_refs as refs
from paper_2603_21090_amd import binding, synth
from tests.helpers import tiny_workload

pytestmark = pytest.mark.gpu


def served_rows():
    w = tiny_workload(num_nodes=60, num_edges=360, batch=60, zipf_s=0.9, layers=2, d_mem=10, d_edge=6, d_time=8, d_msg=10, k=5, heads=2, d_emb=20)
    st = synth.EdgeStream(w)
    g = binding.StreamTGN.from_workload(w, synth.make_weights(w), synth.node_features(w))
    for b in range(6):
        g.ingest_batch(*st.batch(b))
    rows = torch.from_numpy(g.get_embeddings(np.arange(w.num_nodes, dtype=np.uint32)))
    g.close()
    return rows


def parameters(d, hidden):
    g = torch.Generator().manual_seed(9)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return {"gain": 1 + n(d) / 4, "w1": n(d, hidden) * d ** -0.5, "b1": n(hidden) / 4, "w2": n(hidden, d) * hidden ** -0.5, "b2": n(d) / 4, "out": 1 + n(d) / 4}


def test_a_training_step():
    """z = x + dropout(w2 gelu(w1 norm(x) + b1) + b2), y = norm(z): every gradient against automatic differentiation of the same step in 64 bits."""
    x = served_rows()
    n, d = x.shape
    P = parameters(d, 52)
    dy = torch.randn(n, d, generator=torch.Generator().manual_seed(10))
    p = {k: v.cuda() for k, v in P.items()}
    X, DY, rng = x.cuda(), dy.cuda(), torch.tensor([77, 5], dtype=torch.int64, device="cuda")

    def step():
        u = binding.rms_norm(X, p["gain"])
        a, pre = binding.linear(u, p["w1"], bias=p["b1"], activation="gelu", keep_pre=True)
        z = binding.dropout(binding.linear(a, p["w2"], bias=p["b2"]), 0.2, rng, site=1, residual=X)
        y = binding.rms_norm(z, p["out"])
        dz, dout = binding.rms_norm_grad(DY, z, p["out"])
        da, dw2, db2 = binding.linear_grad(binding.dropout_grad(dz, 0.2, rng, site=1), a, p["w2"])
        du, dw1, db1 = binding.linear_grad(da, u, p["w1"], activation="gelu", pre=pre)
        dx, dgain = binding.rms_norm_grad(du, X, p["gain"], dh=dz)
        return {"y": y, "x": dx, "gain": dgain, "w1": dw1, "b1": db1, "w2": dw2, "b2": db2, "out": dout}
    got = step()

    leaf = {k: v.double().requires_grad_() for k, v in {"x": x, **P}.items()}
    norm = lambda t, g: t / torch.sqrt(t.square().mean(1, keepdim=True) + refs.EPS) * g  # noqa: E731
    mask = refs.kept(n, d, 0.2, 77, 5, 1)
    b = torch.nn.functional.gelu(norm(leaf["x"], leaf["gain"]) @ leaf["w1"] + leaf["b1"]) @ leaf["w2"] + leaf["b2"]
    border = round(0.2 * 65536)
    y = norm(leaf["x"] + torch.where(mask, b * (65536 / (65536 - border)), 0.0), leaf["out"])
    want = dict(zip(leaf, torch.autograd.grad((y * dy.double()).sum(), list(leaf.values()))), y=y.detach())
    # eight operators of sums of at most 60 terms: 8 x 2 x 60 x 2^-24 = 6e-5 of the terms' magnitudes at worst, the sums' norms within a factor of ten
    for name, value in want.items():
        err = (got[name].cpu().double() - value).norm() / value.norm()
        assert err <= 6e-4, f"{name}: {err:.2e}"

    graph = torch.cuda.CUDAGraph()                            # captured with the step's number moved on behind it
    with torch.cuda.graph(graph):
        kept = step()
        rng[1:2].add_(1)
    for turn in range(3):
        eager = step()
        graph.replay()
        torch.cuda.synchronize()
        for name in kept:
            assert torch.equal(kept[name], eager[name]), (turn, name)
    assert rng.tolist() == [77, 8]


@pytest.mark.parametrize("rows", [1, 60])
def test_the_block_in_8_bits(rows):
    """Served in 8 bits: what the steps between are is checked against the definition on the numbers in 8 bits that the operators give, and the
    whole against the block in 64 bits: four operands rounded to 8 bits, half a step of 127 each, errors of a product's terms independent."""
    x = served_rows()[:rows]
    P = parameters(x.shape[1], 52)
    p = {k: v.cuda() for k, v in P.items()}
    (w1, s1), (w2, s2) = (binding.quantize(p[k], columns=True) for k in ("w1", "w2"))
    q, s = binding.rms_norm_i8(x.cuda(), p["gain"])
    a = binding.linear_i8(q, s, w1, s1, bias=p["b1"], activation="gelu")
    assert a.dtype == torch.float32
    t, st = binding.quantize(a)
    y = binding.linear_i8(t, st, w2, s2, bias=p["b2"], residual=x.cuda())
    cpu = lambda *v: [i.cpu() for i in v]  # noqa: E731
    want, bound = refs.linear_i8(*cpu(q, s, w1, s1), P["b1"], "gelu", None, torch.float32)
    assert ((a.cpu().double() - want).abs() <= bound).all()
    assert torch.equal(t.cpu(), refs.eight(a.cpu())[0])
    want, bound = refs.linear_i8(*cpu(t, st, w2, s2), P["b2"], "none", x, torch.float32)
    assert ((y.cpu().double() - want).abs() <= bound).all()
    d = {k: v.double() for k, v in P.items()}
    u = refs.rms_norm(x, None, P["gain"])[0][0]
    whole = torch.nn.functional.gelu(u @ d["w1"] + d["b1"]) @ d["w2"] + d["b2"] + x.double()
    # an operand's error is uniform in half a step, max / 254 sqrt(1/3) of it: 0.0023 of the row's largest, at most 0.0023 x 4.5 of its root mean square here; two
    # products of two operands each: sqrt(4) x 0.0103 = 0.021 of the products' terms, whose sums' norm is the products' own
    assert (y.cpu().double() - whole).norm() <= 0.03 * whole.norm()
