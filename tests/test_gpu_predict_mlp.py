"""Link scores by a head with a hidden layer (stgn_set_predictor_mlp): against 64 bits on the rows that the linear head reads out one
number at a time (a one-hot head gives a row's number exactly), in both modes and through every entry point."""
import ctypes as C

import numpy as np
import pytest
import torch

import operator_refs as refs
from paper_2603_21090_amd import binding, synth
from tests.helpers import tiny_workload

pytestmark = pytest.mark.gpu


def make(**kw):
    w = tiny_workload(**{**dict(num_nodes=120, num_edges=900, batch=90, zipf_s=1.0, layers=2, d_mem=12, d_edge=8, d_time=8, d_emb=12, d_msg=12,
                                heads=2, k=4), **kw})
    st = synth.EdgeStream(w)
    g = binding.StreamTGN.from_workload(w, synth.make_weights(w), synth.node_features(w))
    for b in range(6):
        g.ingest_batch(*st.batch(b))
    s, d, t, _ = st.batch(6)
    return w, g, (torch.from_numpy(s.astype(np.int32)).cuda(), torch.from_numpy(d.astype(np.int32)).cuda(), torch.from_numpy(t + 2.0).cuda())


def pairs_of(w, g, edges, mode):
    out = torch.empty(edges[0].shape[0], 2 * w.d_emb)
    for c in range(2 * w.d_emb):
        g.set_predictor(np.eye(2 * w.d_emb, dtype=np.float32)[c], 0.0)
        out[:, c] = g.predict_batch(*edges, at_edge_time=mode).cpu()
    return out


def head(w, hidden, seed=0):
    r = np.random.default_rng(hidden + seed)
    f = lambda *s: r.standard_normal(s).astype(np.float32)  # noqa: E731
    return f(2 * w.d_emb, hidden) / 4, f(hidden), f(hidden), 0.25


def scores(x, w1, b1, w2, b2, act):
    (h, eh), _ = refs.linear(x, torch.from_numpy(w1), torch.from_numpy(b1), act, None)
    v = torch.from_numpy(w2).double()
    y = h @ v + b2
    err = eh @ v.abs() + 2 * (len(w2) + 1) * refs.U * (h.abs() @ v.abs() + abs(b2))
    return y, refs.rounded(y, err, torch.float32)


@pytest.mark.parametrize("kw", [dict(), dict(layers=1, d_mem=0, d_node=10, heads=1, d_emb=50),
                                dict(num_nodes=40000, zipf_s=0.7, d_emb=20)])            # (with a query cache)
@pytest.mark.parametrize("hidden,act", [(1, "none"), (33, "relu"), (200, "gelu")])
def test_scores_in_both_modes(kw, hidden, act):
    w, g, edges = make(**kw)
    for mode in (False, True):
        x = pairs_of(w, g, edges, mode)
        p = head(w, hidden)
        g.set_predictor_mlp(*p, activation=act)
        got = g.predict_batch(*edges, at_edge_time=mode)
        refs.within(got, scores(x, *p, act), f"mode {mode}")
        host = g.predict_batch(*(t.cpu().numpy() for t in edges), at_edge_time=mode)
        assert np.array_equal(host, got.cpu().numpy())
        assert torch.equal(g.predict_batch_static(*edges, at_edge_time=mode), got)
        few = tuple(t[:5].contiguous() for t in edges)
        refs.within(g.predict_batch(*few, at_edge_time=mode), scores(x[:5], *p, act), "five edges")
    g.close()


@pytest.mark.parametrize("mode", [False, True])
def test_ids_out_of_range_and_scores_over_the_inputs(mode):
    w, g, edges = make()
    p = head(w, 16)
    g.set_predictor_mlp(*p, activation="relu")
    want = g.predict_batch(*edges, at_edge_time=mode)
    bad = (edges[0].clone(), edges[1].clone(), edges[2])
    bad[0][3], bad[1][7] = w.num_nodes, -1
    got = g.predict_batch(*bad, at_edge_time=mode)
    nan = torch.isnan(got).cpu()
    assert nan[3] and nan[7] and nan.sum() == 2
    assert torch.equal(got[~nan.cuda()], want[~nan.cuda()])
    ts = edges[2].clone()
    over = ts.view(torch.float32)[:ts.shape[0]]
    g.predict_batch_static(edges[0], edges[1], ts, at_edge_time=mode, out=over)
    assert torch.equal(over, want)
    g.close()


def test_the_last_head_set_is_the_one_that_scores():
    w, g, edges = make()
    lin = np.linspace(-1, 1, 2 * w.d_emb, dtype=np.float32)
    g.set_predictor(lin, 0.5)
    first = g.predict_batch(*edges)
    g.set_predictor_mlp(*head(w, 8))
    a = g.predict_batch(*edges)
    g.set_predictor_mlp(*head(w, 8, seed=1))
    b = g.predict_batch(*edges)
    assert not torch.equal(a, first) and not torch.equal(a, b)
    g.set_predictor(lin, 0.5)
    assert torch.equal(g.predict_batch(*edges), first)
    g.close()


@pytest.mark.parametrize("mode", [False, True])
def test_a_captured_call_follows_the_state(mode):
    w, g, edges = make()
    side = torch.cuda.Stream()
    out = torch.zeros(edges[0].shape[0], device="cuda")
    with torch.cuda.stream(side):
        st = synth.EdgeStream(w)
        h = binding.StreamTGN.from_workload(w, synth.make_weights(w), synth.node_features(w), stream=side)
        for b in range(6):
            h.ingest_batch(*st.batch(b))
        h.set_predictor_mlp(*head(w, 40), activation="silu")
        h.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            h.predict_batch_static(*edges, at_edge_time=mode, out=out)
        for b in range(6, 9):
            graph.replay()
            side.synchronize()
            got = out.clone()
            assert torch.equal(got, h.predict_batch(*edges, at_edge_time=mode))
            h.ingest_batch(*st.batch(b))
            h.sync()
    h.close()
    g.close()


def test_captured_heads_keep_their_width_and_take_new_parameters():
    w, g, edges = make()
    side = torch.cuda.Stream()
    out = torch.zeros(edges[0].shape[0], device="cuda")
    with torch.cuda.stream(side):
        st = synth.EdgeStream(w)
        h = binding.StreamTGN.from_workload(w, synth.make_weights(w), synth.node_features(w), stream=side)
        for b in range(6):
            h.ingest_batch(*st.batch(b))
        h.set_predictor_mlp(*head(w, 24))
        first = h.predict_batch(*edges)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            h.predict_batch_static(*edges, out=out)
        h.set_predictor_mlp(*head(w, 100))                    # another width: the captured one's parameters stay
        filler = [torch.full((1 << 16,), float("nan"), device="cuda") for _ in range(8)]
        for _ in range(3):
            graph.replay()
            side.synchronize()
            assert torch.equal(out, first)
        h.set_predictor_mlp(*head(w, 24, seed=5))             # the same: new ones
        want = h.predict_batch(*edges)
        graph.replay()
        side.synchronize()
        assert torch.equal(out, want) and not torch.equal(out, first)
        del filler
    h.close()
    g.close()


def test_refusals():
    w, g, _ = make()
    L, h = binding.load_library(), g._h
    n = C.c_size_t(0)
    assert L.stgn_predictor_mlp_workspace(h, 0, C.byref(n)) == -1 and L.stgn_predictor_mlp_workspace(h, 4097, C.byref(n)) == -1
    assert L.stgn_predictor_mlp_workspace(h, 8, None) == -1 and L.stgn_predictor_mlp_workspace(h, 8, C.byref(n)) == 0
    w1, b1, w2, _ = head(w, 8)
    p = [binding._ptr(a) for a in (w1, b1, w2)]
    ws = torch.empty(n.value + 256, dtype=torch.uint8, device="cuda")
    at = (ws.data_ptr() + 255) & ~255
    good = [h, 8, 1, *p, 0.0, at, n.value]
    for i, v, code in [(1, 0, -1), (1, 4097, -1), (2, 4, -1), (3, None, -1), (4, None, -1), (5, None, -1), (7, None, -8), (7, at + 16, -8), (8, n.value - 1, -8)]:
        args = list(good)
        args[i] = v
        assert L.stgn_set_predictor_mlp(*args) == code and g.last_error()
    with pytest.raises(binding.StgnError):
        g.predict_batch(np.zeros(1, np.uint32), np.ones(1, np.uint32), np.ones(1))             # no head yet
    g.close()


def test_captured_heads_keep_their_activation():
    """A head of the same width with another activation, set after a capture: the captured one's parameters stay."""
    w, g, edges = make()
    g.close()
    side = torch.cuda.Stream()
    out = torch.zeros(edges[0].shape[0], device="cuda")
    with torch.cuda.stream(side):
        st = synth.EdgeStream(w)
        h = binding.StreamTGN.from_workload(w, synth.make_weights(w), synth.node_features(w), stream=side)
        for b in range(6):
            h.ingest_batch(*st.batch(b))
        h.set_predictor_mlp(*head(w, 24), activation="relu")
        first = h.predict_batch(*edges)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            h.predict_batch_static(*edges, out=out)
        h.set_predictor_mlp(*head(w, 24, seed=3), activation="silu")
        other = h.predict_batch(*edges)
        for _ in range(3):
            graph.replay()
            side.synchronize()
            assert torch.equal(out, first)
        assert torch.equal(h.predict_batch(*edges), other) and not torch.equal(other, first)
    h.close()


def test_a_head_set_while_another_stream_is_current():
    """Memory that the current stream has given back, with work of that stream on it still to come, is not where the head's parameters go."""
    w, g, edges = make()
    _, other, _ = make()
    p = head(w, 64)
    other.set_predictor_mlp(*p, activation="silu")
    want = other.predict_batch(*edges)
    n = C.c_size_t(0)
    assert binding.load_library().stgn_predictor_mlp_workspace(g._h, 64, C.byref(n)) == 0
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        given_back = torch.empty(n.value + 256, dtype=torch.uint8, device="cuda")
        torch.cuda._sleep(1 << 24)
        given_back.fill_(255)
        del given_back
        g.set_predictor_mlp(*p, activation="silu")
    torch.cuda.synchronize()
    assert torch.equal(g.predict_batch(*edges), want)
    g.close()
    other.close()
