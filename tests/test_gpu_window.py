"""Windowed attention, forward and backward, against its definition in 64 bits (window_ref.py derives the bounds)."""
import pytest
import torch

import window_ref as ref
from paper_2505_13389_amd import window

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16
# left, right, sinks, unit
MASKS = {"causal": (-1, 0, 0, 1), "all": (-1, -1, 0, 1), "token_window": (20, 0, 4, 1), "both_sides": (33, 17, 3, 1), "itself": (0, 0, 0, 1),
         "frames": (1, 0, 1, 50), "frames_ahead": (2, 1, 2, 37), "wide_sinks": (3, 0, 130, 1), "many_sinks": (5, 0, 9, 64)}


def tensors(seed, nq, nk, H, Hkv, d, t):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    return (r(nq, H, d)).to(t), (r(nk, Hkv, d) + 0.3 * r(Hkv, d)).to(t), r(nk, Hkv, d).to(t), r(nq, H, d).to(t)


def check_sequences(got, x, lens, mask, dtype, backward=True, scale=None):
    """Packed results against the definition, sequence by sequence."""
    q, k, v, do = x
    a = b = 0
    for nq, nk in lens:
        want = ref.attention(q[a:a + nq], k[b:b + nk], v[b:b + nk], ref.visible(nq, nk, *mask), do[a:a + nq] if backward else None, scale)
        for n, (value, off) in want.items():
            s = (slice(None), slice(a, a + nq)) if n == "lse" else slice(b, b + nk) if n in ("dk", "dv") else slice(a, a + nq)
            ref.check(got[n][s], (value, off), f"{n} of a sequence of {nq} queries, {nk} keys")
        a, b = a + nq, b + nk


def run_packed(x, lens, H, Hkv, d, mask, dtype, scale=0.0, extra=0):
    """Through WindowBuffers, `extra` rows behind the last sequence."""
    left, right, sinks, unit = mask
    q, k, v, do = (t.cuda() for t in x)
    pad = lambda t: torch.cat([t, torch.full((extra, *t.shape[1:]), float("nan"), dtype=t.dtype, device="cuda")])
    q, k, v, do = map(pad, (q, k, v, do))
    cu = lambda i: torch.tensor([sum(l[i] for l in lens[:b]) for b in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    pb = window.WindowProblem(len(lens), H, Hkv, d, max(l[0] for l in lens), max(l[1] for l in lens), left, right, sinks, unit, scale, dtype,
                              q.shape[0], k.shape[0])
    buf = window.WindowBuffers(pb)
    for n in ("out", "lse", "dq", "dk", "dv"):
        getattr(buf, n).fill_(7.0)
    buf.forward(q, k, v, cu(0), cu(1))
    buf.backward(q, k, v, do, cu(0), cu(1))
    torch.cuda.synchronize()
    got = {n: getattr(buf, n).cpu() for n in ("out", "lse", "dq", "dk", "dv")}
    for n in ("out", "dq", "dk", "dv"):
        if extra:
            assert (got[n][-extra:] == 7.0).all(), f"{n}: rows behind the last sequence were written"
    return got


@pytest.mark.parametrize("mask", MASKS.values(), ids=MASKS.keys())
@pytest.mark.parametrize("d,H,Hkv,dtype", [(64, 2, 2, BF), (128, 4, 2, BF), (128, 3, 1, FP), (64, 5, 1, FP)])
def test_packed_sequences(mask, d, H, Hkv, dtype):
    lens = [(1, 1), (200, 200), (0, 0), (63, 63), (1, 130), (65, 300), (0, 5), (100, 0), (3, 3), (90, 40)]
    x = tensors(1, sum(l[0] for l in lens), sum(l[1] for l in lens), H, Hkv, d, dtype)
    got = run_packed(x, lens, H, Hkv, d, mask, dtype, extra=3)
    check_sequences(got, x, lens, mask, dtype)


@pytest.mark.parametrize("n", [1, 31, 32, 33, 64, 127, 129, 511])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths(n, d):
    mask = (40, 0, 2, 1)
    x = tensors(n, n, n, 2, 1, d, BF)
    check_sequences(run_packed(x, [(n, n)], 2, 1, d, mask, BF, scale=0.11), x, [(n, n)], mask, BF, scale=0.11)


@pytest.mark.parametrize("d,dtype", [(64, BF), (128, BF), (128, FP)])
def test_launches_with_a_wavefront_a_block(d, dtype):
    """More blocks than a launch shares among wavefronts."""
    lens = [(193, 193)] * 11
    mask = (70, 0, 3, 1)
    H, Hkv = 16, 16
    x = tensors(5, 193 * 11, 193 * 11, H, Hkv, d, dtype)
    check_sequences(run_packed(x, lens, H, Hkv, d, mask, dtype), x, lens, mask, dtype)


@pytest.mark.parametrize("d,dtype", [(64, FP), (128, BF)])
@pytest.mark.parametrize("mask", [(-1, 0, 0, 1), (-1, -1, 0, 1), (900, 0, 70, 1), (3, 1, 1, 256)])
def test_few_queries_of_many_keys(mask, d, dtype):
    """A walk in several parts, joined; the longest sequence's queries see far more than the others', of which some see nothing."""
    lens = [(40, 3100), (1, 2), (70, 0), (64, 2500), (130, 1)]
    x = tensors(21, sum(l[0] for l in lens), sum(l[1] for l in lens), 2, 1, d, dtype)
    check_sequences(run_packed(x, lens, 2, 1, d, mask, dtype, extra=2), x, lens, mask, dtype)


def test_few_queries_of_many_keys_dense():
    B, H, Hkv, d, mask = 2, 4, 2, 128, (-1, 0, 0, 1)
    lens = [(33, 2100)] * B
    x = tensors(22, 33 * B, 2100 * B, H, Hkv, d, BF)
    q, k, v, do = (t.cuda().unflatten(0, (B, -1)) for t in x)
    pb = window.WindowProblem(B, H, Hkv, d, 33, 2100, *mask)
    buf = window.WindowBuffers(pb)
    buf.forward(q, k, v)
    buf.backward(q, k, v, do)
    got = {n: getattr(buf, n).flatten(0, 1) for n in ("out", "dq", "dk", "dv")}
    check_sequences(got | {"lse": buf.lse}, x, lens, mask, BF)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mask", [(-1, 0, 0, 1), (20, 0, 9, 1), (1, 0, 1, 150)])
@pytest.mark.parametrize("packed", [False, True])
def test_key_blocks_that_many_queries_see(mask, d, packed):
    """Walks of key blocks in parts (long ones, and those of sinks), the heads of a group behind each other."""
    lens, H, Hkv = [(1500, 1500)], 4, 1
    if packed:
        lens = [(1500, 1500), (10, 900), (200, 64)]
    x = tensors(23, sum(l[0] for l in lens), sum(l[1] for l in lens), H, Hkv, d, BF)
    if packed:
        check_sequences(run_packed(x, lens, H, Hkv, d, mask, BF, extra=1), x, lens, mask, BF)
        return
    pb = window.WindowProblem(1, H, Hkv, d, 1500, 1500, *mask)
    buf = window.WindowBuffers(pb)
    q, k, v, do = (t.cuda()[None] for t in x)
    buf.forward(q, k, v)
    buf.backward(q, k, v, do)
    check_sequences({n: getattr(buf, n)[0] for n in ("out", "dq", "dk", "dv")} | {"lse": buf.lse}, x, lens, mask, BF)


def test_many_short_sequences():
    """More sequences than a wavefront has lanes, among them empty ones."""
    lens = [(i * 7 % 67, i * 5 % 71) for i in range(150)]
    mask, H, Hkv, d = (9, 2, 3, 1), 2, 2, 64
    x = tensors(24, sum(l[0] for l in lens), sum(l[1] for l in lens), H, Hkv, d, BF)
    check_sequences(run_packed(x, lens, H, Hkv, d, mask, BF, extra=1), x, lens, mask, BF)


@pytest.mark.parametrize("nq,nk", [(0, 70), (70, 0), (0, 0)])
@pytest.mark.parametrize("packed", [False, True])
def test_no_queries_or_no_keys(nq, nk, packed):
    B, H, Hkv, d = 2, 4, 2, 128
    if packed:
        pb = window.WindowProblem(B, H, Hkv, d, nq, nk, -1, 0, total_q=B * nq, total_k=B * nk)
        cu = [torch.arange(B + 1, dtype=torch.int32, device="cuda") * n for n in (nq, nk)]
        new = lambda n, h: torch.ones(B * n, h, d, dtype=BF, device="cuda")
    else:
        pb, cu = window.WindowProblem(B, H, Hkv, d, nq, nk, -1, 0), [None, None]
        new = lambda n, h: torch.ones(B, n, h, d, dtype=BF, device="cuda")
    buf = window.WindowBuffers(pb, packed=packed)
    for n in ("out", "lse", "dq", "dk", "dv"):
        getattr(buf, n).fill_(7.0)
    q, k, v, do = new(nq, H), new(nk, Hkv), new(nk, Hkv), new(nq, H)
    buf.forward(q, k, v, *cu)
    buf.backward(q, k, v, do, *cu)
    for n in ("out", "dq", "dk", "dv"):
        assert not getattr(buf, n).any(), n
    assert (buf.lse == float("-inf")).all()


def test_two_calls_at_once():
    """Two streams, each with its own buffers, the parts of both in flight together."""
    H, Hkv, d, mask = 4, 1, 128, (-1, 0, 0, 1)
    pb = window.WindowProblem(1, H, Hkv, d, 700, 1500, *mask)
    xs = [[t.cuda()[None] for t in tensors(30 + i, 700, 1500, H, Hkv, d, BF)] for i in range(2)]
    bufs, wants = [window.WindowBuffers(pb) for _ in xs], []
    for x in xs:
        bufs[0].forward(*x[:3])
        bufs[0].backward(*x)
        wants.append({n: getattr(bufs[0], n).clone() for n in ("out", "lse", "dq", "dk", "dv")})
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(5):
        for x, buf, s in zip(xs, bufs, streams):
            with torch.cuda.stream(s):
                buf.forward(*x[:3])
                buf.backward(*x)
    torch.cuda.synchronize()
    for buf, want in zip(bufs, wants):
        for n, t in want.items():
            assert torch.equal(getattr(buf, n), t), n


def test_two_graphs_share_a_workspace():
    """Replayed in turn on one stream: neither leaves anything in the workspace that the other needs."""
    H, Hkv, d = 4, 1, 64
    work, steps = None, []
    for i, (n, mask) in enumerate([(900, (-1, 0, 0, 1)), (300, (50, 0, 3, 1))]):
        pb = window.WindowProblem(1, H, Hkv, d, n, n, *mask)
        x = [t.cuda()[None] for t in tensors(40 + i, n, n, H, Hkv, d, BF)]
        if work is None:
            work = torch.empty(window.vsa_window_workspace_bytes(pb, True), dtype=torch.uint8, device="cuda")
        out, dq, dk, dv = (torch.zeros_like(t) for t in (x[0], x[0], x[1], x[1]))
        lse = torch.zeros(H, n, device="cuda")

        def step(pb=pb, x=x, out=out, lse=lse, grads=(dq, dk, dv)):
            window.vsa_window_forward(pb, *x[:3], out, lse, workspace=work)
            window.vsa_window_backward(pb, *x[:3], out, x[3], lse, *grads, work)
        step()
        torch.cuda.synchronize()
        results = (out, lse, dq, dk, dv)
        want = [t.clone() for t in results]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        steps.append((graph, results, want, x))  # (a graph does not keep its inputs)
    for _ in range(4):
        for graph, results, *_ in steps:
            for t in results:
                t.fill_(3.0)
            graph.replay()
        torch.cuda.synchronize()
        for _, results, want, _ in steps:
            for t, w in zip(results, want):
                assert torch.equal(t, w)


@pytest.mark.parametrize("layout", ["tokens", "heads", "fused", "sliced"])
def test_dense_strides(layout):
    B, L, H, Hkv, d, mask = 3, 150, 4, 2, 128, (1, 0, 1, 30)
    x = tensors(9, B * L, B * L, H, Hkv, d, BF)
    q, k, v, do = (t.cuda().unflatten(0, (B, L)) for t in x)
    if layout == "heads":
        q, k, v, do = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v, do))
    elif layout == "fused":
        qkv = torch.cat([q, k, v], 2)
        q, k, v = qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:]
    elif layout == "sliced":
        wide = lambda t: torch.nn.functional.pad(t, (0, 8, 0, 1, 0, 2))[:, :-2, :-1, :-8]
        q, k, v, do = map(wide, (q, k, v, do))
    pb = window.WindowProblem(B, H, Hkv, d, L, L, *mask)
    buf = window.WindowBuffers(pb)
    buf.forward(q, k, v)
    buf.backward(q, k, v, do)
    got = {n: getattr(buf, n).flatten(0, 1) for n in ("out", "dq", "dk", "dv")}
    got["lse"] = buf.lse
    check_sequences(got, x, [(L, L)] * B, mask, BF)
    # results into strided tensors
    out2, dq2 = torch.zeros(B, H, L, d, dtype=BF, device="cuda").transpose(1, 2), torch.zeros(B, L, H, 2 * d, dtype=BF, device="cuda")[..., :d]
    dk2, dv2 = (torch.zeros(B, L, 2 * Hkv, d, dtype=BF, device="cuda")[:, :, i::2] for i in range(2))
    window.vsa_window_forward(pb, q, k, v, out2)
    window.vsa_window_backward(pb, q, k, v, out2, do, buf.lse, dq2, dk2, dv2, buf.workspace)
    for n, t in (("out", out2), ("dq", dq2), ("dk", dk2), ("dv", dv2)):
        assert torch.equal(t, getattr(buf, n)), n


def test_offsets_past_32_bits():
    L, H, d, mask = 4500, 1, 64, (60, 0, 2, 1)
    x = tensors(3, L, L, H, H, d, BF)
    store = torch.empty(L << 18, dtype=BF, device="cuda")  # rows 2^18 elements apart: 2.4 GB
    far = [store.as_strided((1, L, H, d), (0, 1 << 18, d, 1), 64 * i) for i in range(4)]
    for t, y in zip(far, x):
        t.copy_(y.cuda()[None])
    pb = window.WindowProblem(1, H, H, d, L, L, *mask)
    near, buf = window.WindowBuffers(pb), window.WindowBuffers(pb)
    near.forward(*(y.cuda()[None] for y in x[:3]))
    near.backward(*(y.cuda()[None] for y in x))
    buf.forward(*far[:3])
    buf.backward(*far)
    for n in ("out", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(near, n), getattr(buf, n)), n
    part = slice(L - 300, L)  # and the far end against the definition
    want = ref.attention(x[0][part], x[1], x[2], ref.visible(300, L, *mask))
    ref.check(buf.out[0][part], want["out"], "out")


def test_large_logits_move_the_reference():
    """Logits that grow along the keys: the softmax's reference moves, also in the middle of the walk."""
    n, d = 400, 128
    q, k, v, do = tensors(4, n, n, 1, 1, d, BF)
    k = (k * torch.linspace(0.05, 1.5, n)[:, None, None]).to(BF)
    q = (q * 1.5).to(BF)
    mask = (-1, -1, 0, 1)
    got = run_packed((q, k, v, do), [(n, n)], 1, 1, d, mask, BF)
    check_sequences(got, (q, k, v, do), [(n, n)], mask, BF)
    # very large ones: one key a row counts
    k2 = (k * 40).to(BF)
    got = run_packed((q, k2, v, do), [(n, n)], 1, 1, d, mask, BF)
    s = (q[:, 0].double() @ k2[:, 0].double().t()) / d ** 0.5
    clear = (s.topk(2, 1).values @ torch.tensor([1.0, -1.0], dtype=torch.float64)) > 20
    assert clear.sum() > 50
    assert torch.equal(got["out"][clear, 0], v[s.argmax(1), 0][clear])


def test_same_bits_every_time_and_on_another_stream():
    lens, H, Hkv, d, mask = [(300, 300), (77, 130)], 4, 2, 128, (30, 0, 2, 1)
    x = tensors(6, 377, 430, H, Hkv, d, BF)
    first = run_packed(x, lens, H, Hkv, d, mask, BF)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run_packed(x, lens, H, Hkv, d, mask, BF)
    side.synchronize()
    for n in first:
        assert torch.equal(first[n], again[n]), n


def test_captured_and_replayed():
    B, L, H, d, mask = 1, 333, 2, 128, (2, 0, 1, 40)
    pb = window.WindowProblem(B, H, H, d, L, L, *mask)
    eager, graphed = window.WindowBuffers(pb), window.WindowBuffers(pb)
    x = [t.cuda()[None] for t in tensors(0, L, L, H, H, d, BF)]

    def step(buf):
        buf.forward(*x[:3])
        buf.backward(*x)
    step(graphed)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    for seed in range(4):
        for t, y in zip(x, tensors(seed, L, L, H, H, d, BF)):
            t.copy_(y[None])
        step(eager)
        graph.replay()
        torch.cuda.synchronize()
        for n in ("out", "lse", "dq", "dk", "dv"):
            assert torch.equal(getattr(eager, n), getattr(graphed, n)), (seed, n)


def test_offsets_that_lie_stay_in_bounds():
    """Offsets outside the tensors, falling or longer than announced are clamped: neighbours of the tensors stay as they were."""
    H, d, rows = 2, 64, 100
    x = [torch.randn(rows + 128, H, d, device="cuda").to(BF) for _ in range(4)]
    q, k, v, do = (t[64:64 + rows] for t in x)
    pb = window.WindowProblem(3, H, H, d, 50, 50, 10, 0, 1, 1, total_q=rows, total_k=rows)
    cu = torch.tensor([-40, 70, 20, 5000], dtype=torch.int32, device="cuda")
    outs = [torch.full((rows + 128, H, d), 3.0, dtype=BF, device="cuda") for _ in range(4)]
    lse = torch.zeros(H, rows, device="cuda")
    ws = torch.empty(window.vsa_window_workspace_bytes(pb, True), dtype=torch.uint8, device="cuda")
    mid = [t[64:64 + rows] for t in outs]
    window.vsa_window_forward(pb, q, k, v, mid[0], lse, cu, cu)
    window.vsa_window_backward(pb, q, k, v, mid[0], do, lse, *mid[1:], ws, cu, cu)
    torch.cuda.synchronize()
    for t in outs:
        assert (t[:64] == 3.0).all() and (t[64 + rows:] == 3.0).all()
    want = ref.attention(q[:50].cpu(), k[:50].cpu(), v[:50].cpu(), ref.visible(50, 50, 10, 0, 1, 1))  # the first: rows 0 to 49
    value, off = want["out"]  # ... of which the third, rows 20 (its own offset) to 69, has 20 to 49 too
    ref.check(mid[0][:20], (value[:20], off[:20]), "out")


def test_gradient_against_differences():
    """The formula of the backward against central differences of the forward's definition in 64 bits."""
    mask, n, H, Hkv, d = (6, 1, 2, 3), 24, 4, 2, 64
    x = tensors(8, n, n, H, Hkv, d, BF)
    got = run_packed(x, [(n, n)], H, Hkv, d, mask, BF)
    see = ref.visible(n, n, *mask)
    loss = lambda q, k, v: float((ref.attention(q, k, v, see, out_type=BF)["out"][0] * x[3].double()).sum())
    g = torch.Generator().manual_seed(2)
    for i, name in enumerate(("dq", "dk", "dv")):
        want = ref.attention(*x[:3], see, x[3])[name]
        for _ in range(4):
            way = torch.randn(x[i].shape, generator=g, dtype=torch.float64)
            at = [t.double() for t in x[:3]]
            h = 1e-5
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * way, at[i] - h * way
            slope = (loss(*up) - loss(*down)) / (2 * h)
            assert abs(slope - float((want[0] * way).sum())) <= 1e-6 * (1 + abs(slope))
            assert abs(slope - float((got[name].double() * way).sum())) <= float((want[1] * way.abs()).sum()) + 1e-6 * (1 + abs(slope))


def op_case():
    lens = [(70, 70), (1, 1), (130, 200)]
    x = tensors(11, sum(l[0] for l in lens), sum(l[1] for l in lens), 4, 2, 64, FP)
    cu = [torch.tensor([0, *torch.tensor([l[i] for l in lens]).cumsum(0).tolist()], dtype=torch.int32, device="cuda") for i in (0, 1)]
    return lens, x, cu


def test_autograd_packed():
    from paper_2505_13389_amd.autograd import window_attention
    lens, x, (cu_q, cu_k) = op_case()
    mask = (30, 0, 4, 1)
    q, k, v = (t.cuda().requires_grad_() for t in x[:3])
    out = window_attention(q, k, v, left=30, sinks=4, cu_q=cu_q, cu_k=cu_k, max_q=130, max_k=200)
    out.backward(x[3].cuda())
    check_sequences({"out": out.detach(), "dq": q.grad, "dk": k.grad, "dv": v.grad, "lse": torch.cat([ref.attention(
        x[0][a:a + n], x[1][b:b + m], x[2][b:b + m], ref.visible(n, m, *mask))["lse"][0] for a, b, (n, m) in
        zip(cu_q.tolist(), cu_k.tolist(), lens)], 1)}, x, lens, mask, FP)


def test_autograd_of_shared_and_broadcast_inputs():
    """Keys and values that batches share (expanded, stride 0), rows that are not 16-byte aligned, a gradient that is broadcast."""
    from paper_2505_13389_amd.autograd import window_attention
    B, L, H, d, mask = 2, 90, 2, 64, (1, 0, 1, 16)
    q, k, v, _ = tensors(12, L, L, H, H, d, BF)
    store = torch.zeros(L * H * d + 1, dtype=BF, device="cuda")
    store[1:] = k.cuda().flatten()
    kk = store[1:].view(L, H, d).requires_grad_()
    qq, vv = q.cuda().requires_grad_(), v.cuda().requires_grad_()
    expand = lambda t: t[None].expand(B, -1, -1, -1)
    out = window_attention(expand(qq), expand(kk), expand(vv), left=1, sinks=1, unit=16)
    out.sum().backward()
    want = ref.attention(q, k, v, ref.visible(L, L, *mask), torch.ones(L, H, d, dtype=BF))
    for n, t in (("dq", qq), ("dk", kk), ("dv", vv)):
        value, off = want[n]  # summed over the batches: twice the value, rounded once more
        ref.check(t.grad, (2 * value, 2 * off + 2 * value.abs() * ref.HALF[BF]), n)


def test_autograd_captured_and_replayed():
    """Captured where no eager graph of the leaves lives; refused where one does (its gradient nodes would tie the capture to
    an uncaptured stream)."""
    from paper_2505_13389_amd.autograd import window_attention
    B, L, H, d = 1, 100, 2, 64
    q, k, v = (t.cuda()[None].requires_grad_() for t in tensors(13, L, L, H, H, d, BF)[:3])
    do = torch.randn(B, L, H, d, device="cuda").to(BF)
    call = lambda: window_attention(q, k, v, left=20, sinks=2)
    want = torch.autograd.grad(call(), (q, k, v), do)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = torch.autograd.grad(call(), (q, k, v), do)
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
