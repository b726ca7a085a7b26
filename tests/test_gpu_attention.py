"""Attention of lists and its gradients against 64 bits (bounds: operator_refs)."""
import pytest
import torch

import operator_refs as refs
from paper_2603_21090_amd import binding

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# lists, q_len, k_len, heads, kv_heads, d, causal, window, ragged
SHAPES = [
    (1, 1, 1, 1, 1, 1, False, 0, False), (1, 1, 1, 2, 1, 64, True, 0, False), (7, 1, 10, 2, 2, 50, False, 0, True),
    (40, 1, 20, 2, 2, 50, False, 0, True), (5, 1, 33, 4, 1, 25, False, 0, True), (3, 1, 64, 1, 1, 256, False, 0, True),
    (2, 1, 700, 8, 2, 128, False, 0, True), (1, 1, 5000, 4, 4, 32, True, 0, False), (2, 1, 3001, 16, 1, 80, False, 0, True),
    (2, 3, 300, 4, 2, 64, True, 0, True), (2, 5, 130, 6, 2, 40, True, 7, True), (3, 17, 17, 2, 2, 16, True, 0, True),
    (2, 65, 65, 4, 2, 100, True, 0, True), (2, 100, 37, 2, 1, 64, True, 0, True), (2, 37, 100, 2, 1, 33, True, 20, True),
    (1, 200, 200, 3, 3, 128, True, 0, False), (1, 200, 200, 3, 1, 96, False, 0, False), (2, 130, 190, 2, 2, 7, False, 0, True),
    (2, 150, 150, 4, 1, 72, True, 1, True), (1, 300, 300, 2, 1, 64, True, 64, True), (1, 70, 90, 1, 1, 200, True, 0, True),
    (1, 129, 257, 2, 2, 256, False, 0, True), (2, 90, 20, 8, 1, 40, True, 5, True), (1, 3, 400, 24, 2, 48, True, 9, False),
    (1, 20, 30, 16, 1, 100, True, 0, False), (2, 70, 300, 10, 2, 130, True, 50, True), (1, 2, 1500, 40, 1, 64, True, 0, False),
    (1, 700, 9, 4, 2, 33, False, 0, False), (1, 5, 2500, 8, 2, 80, True, 600, True),
]


def make(lists, ql, kl, heads, kv, d, ragged, dt, seed=0):
    g = torch.Generator().manual_seed(hash((lists, ql, kl, heads, d)) % (1 << 31) + seed)
    n = lambda *s: torch.randn(*s, generator=g).to(dt)  # noqa: E731
    q, k, v, do = n(lists, ql, heads, d), n(lists, kl, kv, d), n(lists, kl, kv, d), n(lists, ql, heads, d)
    if not ragged:
        return q, k, v, do, None, None
    qn = torch.randint(0, ql + 1, (lists,), generator=g, dtype=torch.int32) if ql > 1 else torch.ones(lists, dtype=torch.int32)
    kn = torch.randint(0, kl + 1, (lists,), generator=g, dtype=torch.int32)
    kn[0], qn[0] = kl, ql                                     # the longest is there; the last one is empty where there are enough
    if lists > 4:
        kn[-1] = 0
    for b in range(lists):                                    # nobody reads what lies behind a list's end
        q[b, qn[b]:], do[b, qn[b]:], k[b, kn[b]:], v[b, kn[b]:] = (float("nan"),) * 4
    return q, k, v, do, qn, kn


def on_gpu(*ts):
    return tuple(None if t is None else t.cuda() for t in ts)


def check(q, k, v, do, qn, kn, causal, window, scale=None, prepared=None):
    see = refs.visible(q.shape[0], q.shape[1], k.shape[1], qn, kn, causal, window)
    want = refs.attention(q, k, v, see, q.shape[3] ** -0.5 if scale is None else scale, do)
    Q, K, V, DO, QN, KN = prepared or on_gpu(q, k, v, do, qn, kn)
    kw = dict(q_lens=QN, k_lens=KN, causal=causal, window=window, scale=scale)
    out, lse = binding.attention(Q, K, V, **kw)
    refs.within(out, want["out"], "out")
    refs.within(lse, want["lse"], "lse")
    for name, got in zip(("dq", "dk", "dv"), binding.attention_grad(DO, Q, K, V, out, lse, **kw)):
        refs.within(got, want[name], name)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_gradients(shape, dt):
    lists, ql, kl, heads, kv, d, causal, window, ragged = shape
    check(*make(lists, ql, kl, heads, kv, d, ragged, dt), causal, window)


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_strides_of_heads_first_of_packed_rows_and_of_shared_lists(dt):
    q, k, v, do, _, _ = make(3, 40, 50, 4, 4, 36, False, dt)
    heads_first = lambda t: t.cuda().transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    packed = torch.full((3, 50, 8 * 36 + 5), float("nan"), dtype=dt, device="cuda")   # a row's keys and values and five numbers more, one in
    packed[:, :, 1:289] = torch.cat([k, v], 2).reshape(3, 50, 288).cuda()
    K, V = (packed[:, :, 1 + 144 * x:145 + 144 * x].unflatten(2, (4, 36)) for x in (0, 1))
    check(q, k, v, do, None, None, True, 0, prepared=(heads_first(q), K, V, heads_first(do), None, None))
    shared = lambda t: t[:1].expand(3, -1, -1, -1)            # noqa: E731  one list of keys for all queries
    check(q, shared(k), shared(v), do, None, None, False, 0, prepared=(q.cuda(), shared(k.cuda()), shared(v.cuda()), do.cuda(), None, None))


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_outputs_kept_heads_first(dt):
    q, k, v, do, qn, kn = make(3, 30, 50, 4, 2, 36, True, dt)
    Q, K, V, DO, QN, KN = on_gpu(q, k, v, do, qn, kn)
    out, lse = binding.attention(Q, K, V, q_lens=QN, k_lens=KN)
    kept = out.transpose(1, 2).contiguous().transpose(1, 2)
    for a, b in zip(binding.attention_grad(DO, Q, K, V, out, lse, q_lens=QN, k_lens=KN),
                    binding.attention_grad(DO, Q, K, V, kept, lse, q_lens=QN, k_lens=KN)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("ql", [1, 4, 40])
def test_large_scores_and_other_scales(dt, ql):
    """Scores up to some hundreds: softmax weights of zero and one, nothing overflows; a scale of its own, zero and negative ones."""
    q, k, v, do, qn, kn = make(2, ql, 90, 2, 1, 32, True, dt, seed=7)
    for scale in (4.0, -0.3, 0.0):
        check(q, k, v, do, qn, kn, False, 0, scale=scale)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("ql", [1, 33])
def test_lengths_outside_the_padded_ones_count_as_the_nearer_end(dt, ql):
    q, k, v, do, _, _ = make(4, ql, 20, 2, 2, 24, False, dt)
    kn = torch.tensor([-3, 20, 1000, 5], dtype=torch.int32)
    qn = torch.tensor([ql, 99, -1, ql], dtype=torch.int32)
    Q, K, V, DO = on_gpu(q, k, v, do)
    out, lse = binding.attention(Q, K, V, q_lens=qn.cuda(), k_lens=kn.cuda())
    near = dict(q_lens=qn.clamp(0, ql).cuda(), k_lens=kn.clamp(0, 20).cuda())
    o2, l2 = binding.attention(Q, K, V, **near)
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    for a, b in zip(binding.attention_grad(DO, Q, K, V, out, lse, q_lens=qn.cuda(), k_lens=kn.cuda()),
                    binding.attention_grad(DO, Q, K, V, out, lse, **near)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("lists,ql,kl", [(0, 3, 5), (2, 0, 5), (2, 3, 0), (1, 1, 0)])
def test_nothing_to_do(lists, ql, kl, dt):
    q, k = torch.zeros(lists, ql, 4, 16, dtype=dt, device="cuda"), torch.zeros(lists, kl, 2, 16, dtype=dt, device="cuda")
    out, lse = binding.attention(q, k, k)
    assert not out.any() and torch.isneginf(lse).all()
    dq, dk, dv = binding.attention_grad(q, q, k, k, out, lse)
    assert not dq.any() and not dk.any() and not dv.any()


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("ql,kl", [(1, 2000), (1, 12), (90, 90)])
def test_the_same_bits_again_on_another_stream_and_in_a_graph(dt, ql, kl):
    q, k, v, do, qn, kn = make(3, ql, kl, 4, 2, 64, True, dt)
    q, k, v, do = (torch.nan_to_num(t) for t in (q, k, v, do))
    Q, K, V, DO, QN, KN = on_gpu(q, k, v, do, qn, kn)

    def step():
        out, lse = binding.attention(Q, K, V, q_lens=QN, k_lens=KN, causal=True)
        return (out, lse) + binding.attention_grad(DO, Q, K, V, out, lse, q_lens=QN, k_lens=KN, causal=True)
    first = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    for a, c in zip(first, other):
        assert torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for turn in range(3):
        V.mul_(-1 if turn else 1)
        KN.sub_(turn).clamp_(min=0)
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        for a, c in zip(kept, eager):
            assert torch.equal(a, c)


def test_gradients_against_differences():
    """d/dh of sum(out * dout) along random directions, by central differences of the fp32 kernel itself: steps of 2^-6 leave a
    third-order term (of the order of h^2) and the rounding of two sums of 5,000 numbers of about one, over 2 h."""
    q, k, v, do, qn, kn = make(2, 30, 40, 2, 1, 20, True, torch.float32)
    q, k, v, do = (torch.nan_to_num(t) for t in (q, k, v, do))
    Q, K, V, DO, QN, KN = on_gpu(q, k, v, do, qn, kn)
    kw = dict(q_lens=QN, k_lens=KN, causal=True)
    out, lse = binding.attention(Q, K, V, **kw)
    grads = binding.attention_grad(DO, Q, K, V, out, lse, **kw)
    value = lambda *t: (binding.attention(*t, **kw)[0].double() * DO.double()).sum().item()  # noqa: E731
    g = torch.Generator(device="cuda").manual_seed(3)
    for at in range(3):
        dirn = torch.randn([Q, K, V][at].shape, generator=g, device="cuda")
        slopes = []
        for h in (2.0 ** -6, 2.0 ** -7):
            plus, minus = [Q, K, V], [Q, K, V]
            plus[at], minus[at] = plus[at] + h * dirn, minus[at] - h * dirn
            slopes.append((value(*plus) - value(*minus)) / (2 * h))
        best = (4 * slopes[1] - slopes[0]) / 3                # the h^2 term taken out; what is left is below the two slopes' distance
        noise = 2 * 2.0 ** -24 * 60 * 2.0 ** 7 * 8            # rounding of the weights: u times 60 rows' worth of |out . dout|, over h
        assert abs(best - (grads[at].double() * dirn.double()).sum().item()) <= abs(slopes[0] - slopes[1]) + noise


@pytest.mark.parametrize("ql,kl", [(1, 3000), (200, 200)])
def test_calls_at_the_same_time_on_two_streams(ql, kl):
    """Both in flight, again and again, each with buffers of its own: the bits of a call alone."""
    sides, kept = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for n in range(2):
        q, k, v, do, _, _ = make(4, ql, kl, 4, 2, 64, False, torch.bfloat16, seed=n)
        Q, K, V, DO = on_gpu(q, k, v, do)
        out, lse = binding.attention(Q, K, V, causal=True)
        kept.append((Q, K, V, DO, out, lse, binding.attention_grad(DO, Q, K, V, out, lse, causal=True)))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for n, side in enumerate(sides):
            with torch.cuda.stream(side):
                Q, K, V, DO, out, lse, _ = kept[n]
                got[n].append(binding.attention(Q, K, V, causal=True) + binding.attention_grad(DO, Q, K, V, out, lse, causal=True))
    torch.cuda.synchronize()
    for n in range(2):
        want = (kept[n][4], kept[n][5]) + tuple(kept[n][6])
        for res in got[n]:
            assert all(torch.equal(a, b) for a, b in zip(res, want))


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("lists,kl,kv,group", [(2, 300, 2, 1), (1, 5000, 1, 4), (3, 129, 2, 2)])
def test_no_queries_over_keys(lists, kl, kv, group, dt):
    """Lists of any length without queries: zeros as gradients, nothing else (5,000 and 300 keys are cut into runs, 129 are not)."""
    q = torch.zeros(lists, 0, kv * group, 40, dtype=dt, device="cuda")
    k = torch.ones(lists, kl, kv, 40, dtype=dt, device="cuda")
    out, lse = binding.attention(q, k, k)
    assert out.shape == q.shape and lse.shape == (lists, kv * group, 0)
    dq, dk, dv = binding.attention_grad(q, q, k, k, out, lse)
    assert dq.shape == q.shape and dk.shape == dv.shape == k.shape and not dk.any() and not dv.any()


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("ql,kl,window,kv,d", [(1, 90, 5, 2, 64), (3, 400, 9, 2, 50), (10, 40, 4, 2, 64), (10, 40, 4, 1, 33), (40, 90, 7, 2, 64),
                                               (130, 700, 20, 2, 128), (20, 50, 3, 2, 200)])
def test_masked_keys_hold_the_type_s_largest_numbers(ql, kl, window, kv, d, dt):
    """Keys in front of every query's window hold the largest and the lowest numbers of the type: their products with dout and the queries
    are infinite or not numbers, and belong to no pair that counts."""
    q, k, v, do, _, _ = make(3, ql, kl, 2, kv, d, False, dt)
    kn, qn = torch.tensor([kl, kl - 3, kl - 1], dtype=torch.int32), torch.tensor([ql, max(ql - 2, 1), ql], dtype=torch.int32)
    unseen = ~refs.visible(3, ql, kl, qn, kn, True, window).any(1)
    assert unseen.any(1).all()
    most = torch.finfo(dt).max
    for t in (k, v):
        t[unseen] = most
        t[..., 1::2][unseen] = -most
        t[:, ::2][unseen[:, ::2]] = -most                     # (every other key: sums of one sign)
    check(q, k, v, do, qn, kn, True, window)


def dealt(n, lo, hi):
    """n powers of two from 2^lo up to 2^hi, each about as often."""
    return 2.0 ** torch.linspace(lo, hi, n).round()


# q_len, k_len, scale, exponents of q, k, v and of dout (of all rows, or first to last)
MAGNITUDES = [(24, 4000, 0.125, -6, 6, 0, (-14, -14)),        # dq of ds around fp16's smallest number
              (24, 4000, 0.125, -8, 8, 0, (-18, -18)),        # and below it
              (300, 4000, 0.125, 6, -6, 0, (-14, -14)),       # dk
              (24, 20, 2.0 ** -9, 0, 0, 9, (9, 9)),           # ds above fp16's largest
              (300, 700, 2.0 ** -7, 0, 0, 4, (-14, 9)),       # rows of all magnitudes, growing
              (300, 700, 2.0 ** -7, 0, 0, 4, (9, -14))]       # and shrinking


@pytest.mark.parametrize("ql,kl,scale,eq,ek,ev,edo", MAGNITUDES, ids=str)
@pytest.mark.parametrize("heads,kv,d", [(2, 1, 64), (1, 1, 100), (1, 1, 160)])
def test_half_precision_gradients_of_any_magnitude(ql, kl, scale, eq, ek, ev, edo, heads, kv, d):
    """ds as an fp16 factor keeps its bits whatever its size: one rounding of 2^-11 of each, and 2^-33 of the largest that a sum has met (the
    factors are scaled until that one lies above 2^8, where fp16's last step is 2^-25).  refs grants the factors fp16's smallest step instead:
    taken out here, and for the outputs put back."""
    q, k, v, do, _, _ = make(1, ql, kl, heads, kv, d, False, torch.float32, seed=11)
    q, k, v = q * 2.0 ** eq, k * 2.0 ** ek, v * 2.0 ** ev
    do = do * dealt(ql, *edo)[None, :, None, None]
    q, k, v, do = (t.half() for t in (q, k, v, do))
    see = refs.visible(1, ql, kl, None, None, False, 0)
    kept = refs.TINY[torch.float16]
    try:
        refs.TINY[torch.float16] = 0.0
        want = refs.attention(q, k, v, see, scale, do)
    finally:
        refs.TINY[torch.float16] = kept
    heads_first = lambda t: t.double().permute(0, 2, 1, 3)    # noqa: E731
    Q, DO = heads_first(q), heads_first(do)
    K, V = (heads_first(t).repeat_interleave(heads // kv, 1) for t in (k, v))
    p = torch.softmax(scale * (Q @ K.transpose(2, 3)), -1)
    dp = DO @ V.transpose(2, 3)
    ds = (p * (dp - (p * dp).sum(-1, keepdim=True))).abs()
    step = 2.0 ** -33 * scale
    more = {"dq": (ds.amax(-1, keepdim=True) * K.abs().sum(2, keepdim=True)).permute(0, 2, 1, 3) * step,
            "dk": (ds.amax(2)[..., None] * Q.abs().sum(2, keepdim=True)).permute(0, 2, 1, 3) * step, "dv": 0.0}
    if heads > kv:
        more["dk"] = more["dk"].sum(2, keepdim=True)
    Qg, Kg, Vg, DOg = on_gpu(q, k, v, do)
    out, lse = binding.attention(Qg, Kg, Vg, scale=scale)
    for name, got in zip(("dq", "dk", "dv"), binding.attention_grad(DOg, Qg, Kg, Vg, out, lse, scale=scale)):
        value, bound = want[name]
        assert torch.isfinite(value).all() and value.abs().max() < 65504
        refs.within(got, (value, bound + more[name] + 2 * kept), name)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("ql,kl,heads,kv,d,causal,window", [(60, 9000, 1, 1, 33, False, 0), (9000, 50, 1, 1, 33, False, 0), (30, 8300, 2, 1, 64, True, 0),
                                                            (8800, 60, 2, 1, 40, True, 0), (40, 8200, 1, 1, 130, False, 0)])
def test_runs_of_long_streams(ql, kl, heads, kv, d, causal, window, dt):
    """Few tiles against streams of 8,192 rows and more: sixteen runs and more, joined by the waves of a workgroup."""
    check(*make(1, ql, kl, heads, kv, d, True, dt), causal, window)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("ql,kl", [(1, 300), (2, 60), (40, 90)])
def test_offsets_past_32_bits(ql, kl, dt):
    """Lists 2^31 + 5 numbers apart, or rows so far apart that the last values lie that far behind the first: everything in one buffer."""
    q, k, v, do, qn, kn = make(2, ql, kl, 2, 2, 50, True, dt)
    far = (1 << 31) + 5
    buffer = torch.empty(far + kl * 2 * 50 + 64, dtype=dt, device="cuda")
    lists = buffer.as_strided((2, kl, 2, 50), (far, 100, 50, 1), 3)
    lists.copy_(k.cuda())
    Q, V, DO, QN, KN = on_gpu(q, v, do, qn, kn)
    check(q, k, v, do, qn, kn, True, 0, prepared=(Q, lists, V, DO, QN, KN))
    row = (far - 1000) // kl
    rows = buffer.as_strided((2, kl, 2, 50), (150, row, 50, 1), 3)
    rows.copy_(v.cuda())
    check(q, k, v, do, qn, kn, True, 0, prepared=(Q, k.cuda(), rows, DO, QN, KN))
