"""Host side of windowed attention and the cache (no GPU): how blocks walk, what is refused, what the binding checks."""
import ctypes as C
import random

import pytest
import torch

from paper_2505_13389_amd import vsa, window

BF = torch.bfloat16


@pytest.mark.parametrize("seed", range(8))
def test_walks_visit_every_visible_pair_once(seed):
    r = random.Random(seed)
    for _ in range(12):
        unit = r.choice([1, 1, 2, 7, 50, 64, 100])
        pb = window.WindowProblem(1, 1, 1, 64, 400, 400, r.choice([-1, 0, 1, 3, r.randint(0, 300)]), r.choice([-1, 0, 0, 1, r.randint(0, 90)]),
                                  r.choice([0, 0, 1, 4, r.randint(0, 200)]), unit)
        nq, nk = r.choice([0, 1, 64, r.randint(0, 330)]), r.choice([0, 1, 64, r.randint(0, 330)])
        if r.random() < 0.5:
            nk = nq
        assert window.vsa_host_window_walk(pb, nq, nk) == 0, (pb, nq, nk)


def test_walks_of_the_largest_parameters():
    most = 2 ** 31 - 1
    for left, right, sinks, unit in ((most, most, most, most), (most, 0, 0, 1), (0, most, 0, 3), (0, 0, most, 100), (-1, -1, most, most)):
        assert window.vsa_host_window_walk(window.WindowProblem(1, 1, 1, 64, 99, 99, left, right, sinks, unit), 70, 99) == 0


def params(**k):
    base = dict(B=1, H=2, Hkv=2, d=64, max_q=8, max_k=8)
    base.update(k)
    p = window.WindowProblem(**base).params()
    for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        setattr(p, n, window.VsaStrides(8 * 128, 128, 64))
    return p


FAKE = 1 << 20  # an aligned address that is never touched: every call below is refused first


@pytest.mark.parametrize("change,status", [
    (dict(d=96), -3), (dict(B=0), -2), (dict(H=3), -2), (dict(Hkv=0), -2), (dict(unit=0), -2), (dict(left=-2), -2), (dict(right=-2), -2),
    (dict(sinks=-1), -2), (dict(softmax_scale=float("nan")), -2), (dict(softmax_scale=float("inf")), -2), (dict(max_q=-1), -2),
    (dict(max_q=(1 << 30) + 1), -3), (dict(B=1 << 20, max_q=1 << 10), -3)])
def test_bad_windows_are_refused(change, status):
    p = params(**change)
    L = vsa.lib()
    assert L.vsa_window_forward(C.byref(p), *[FAKE] * 3, None, None, FAKE, None, FAKE, 1 << 40, None) == status
    assert L.vsa_window_backward(C.byref(p), *[FAKE] * 3, None, None, *[FAKE] * 7, 1 << 40, None) == status
    assert L.vsa_window_workspace_bytes(C.byref(p), 0) == 0 and L.vsa_window_workspace_bytes(C.byref(p), 1) == 0


def test_bad_pointers_strides_and_workspaces_are_refused():
    L, p = vsa.lib(), params()
    fwd = lambda q=FAKE, k=FAKE, v=FAKE, cq=None, ck=None, o=FAKE, lse=None, p=p, ws=FAKE, n=1 << 40: L.vsa_window_forward(
        C.byref(p), q, k, v, cq, ck, o, lse, ws, n, None)
    assert L.vsa_window_forward(None, *[None] * 8, 0, None) == -1
    assert fwd(q=None) == -1 and fwd(k=None) == -1 and fwd(v=None) == -1 and fwd(o=None) == -1
    assert fwd(q=FAKE + 8) == -4 and fwd(o=FAKE + 2) == -4 and fwd(lse=FAKE + 2) == -4
    assert fwd(cq=FAKE) == -2 and fwd(ck=FAKE) == -2  # both or neither
    for name, strides, status in (("q", (1024, 132, 64), -4), ("k", (1024, -128, 64), -2), ("v", (1024, 1 << 25, 64), -3),
                                  ("out", (1024, 128, 0), -2), ("out", (1024, 56, 64), -2)):
        x = params()
        setattr(x, name, window.VsaStrides(*strides))
        assert fwd(p=x) == status, name
    need = L.vsa_window_workspace_bytes(C.byref(p), 0)
    assert need > 0 and fwd(ws=None) == -5 and fwd(n=need - 1) == -5 and fwd(ws=FAKE + 4) == -4
    need = L.vsa_window_workspace_bytes(C.byref(p), 1)
    bwd = lambda ws, n: L.vsa_window_backward(C.byref(p), *[FAKE] * 3, None, None, *[FAKE] * 6, ws, n, None)
    assert need >= 2 * 8 * 8 and bwd(None, need) == -5 and bwd(FAKE, need - 1) == -5 and bwd(FAKE + 4, need) == -4


def cache_params(**k):
    base = dict(B=2, H=4, Hkv=2, d=64, max_q=1, total_q=0, pages=4, max_pages=3, unit=1, left=-1, right=0)
    base.update(k)
    p = window.VsaCache(**base)
    for n in ("q", "out"):
        setattr(p, n, window.VsaStrides(256, 256, 64))
    for n in ("k", "v"):
        setattr(p, n, window.VsaStrides(128, 128, 64))
    return p


@pytest.mark.parametrize("change,status", [
    (dict(B=0), -2), (dict(H=3), -2), (dict(d=32), -3), (dict(pages=0), -2), (dict(max_pages=0), -2), (dict(max_pages=1 << 25), -3),
    (dict(unit=0), -2), (dict(left=-3), -2), (dict(sinks=-1), -2), (dict(softmax_scale=float("nan")), -2), (dict(dtype=2), -2), (dict(max_q=-1), -2)])
def test_bad_caches_are_refused(change, status):
    p = cache_params(**change)
    L = vsa.lib()
    assert L.vsa_cache_attention(C.byref(p), FAKE, None, *[FAKE] * 7, None, FAKE, 1 << 40, None) == status
    assert L.vsa_cache_workspace_bytes(C.byref(p)) == 0


def test_bad_pointers_of_caches_are_refused():
    L, p = vsa.lib(), cache_params()
    need = L.vsa_cache_workspace_bytes(C.byref(p))
    good = [FAKE, None, *[FAKE] * 7, None, FAKE, need, None]  # q, cu, lens, table, k, v, k_scale, v_scale, out, lse, workspace
    for at in (0, 2, 3, 4, 5, 6, 7, 8):
        bad = list(good)
        bad[at] = None
        assert L.vsa_cache_attention(C.byref(p), *bad) == -1, at
        bad[at] = FAKE + 2
        assert L.vsa_cache_attention(C.byref(p), *bad) == -4, at
    assert L.vsa_cache_attention(C.byref(p), *good[:10], None, need, None) == -5
    assert L.vsa_cache_attention(C.byref(p), *good[:10], FAKE, need - 1, None) == -5
    app = [FAKE, FAKE, None, *[FAKE] * 6, None]  # k, v, cu, lens, table, pages and scales
    for at in (0, 1, 3, 4, 5, 6, 7, 8):
        bad = list(app)
        bad[at] = None
        assert L.vsa_cache_append(C.byref(p), *bad) == -1, at
    assert L.vsa_cache_append(C.byref(cache_params(Hkv=0)), *app) == -2
    q = cache_params()
    q.out = window.VsaStrides(256, 256, 0)
    assert L.vsa_cache_attention(C.byref(q), *good) == -2


def test_the_binding_checks_shapes_types_and_devices():
    pb = window.WindowProblem(1, 2, 1, 64, 4, 6)
    t = lambda *s, dtype=BF: torch.zeros(*s, dtype=dtype)
    q, k, o = t(1, 4, 2, 64), t(1, 6, 1, 64), t(1, 4, 2, 64)
    for bad in ((t(1, 5, 2, 64), k, k, o), (q, t(1, 6, 2, 64), k, o), (q, k, t(1, 6, 1, 64, dtype=torch.float16), o), (q, k, k, t(1, 4, 2, 63)),
                (q, k, t(1, 6, 64, 1).transpose(2, 3), o)):
        with pytest.raises(ValueError):
            window.vsa_window_forward(pb, *bad)
    with pytest.raises(ValueError, match="on a GPU"):
        window.vsa_window_forward(pb, q, k, k, o)
    with pytest.raises(ValueError, match="both or neither"):
        window.vsa_window_forward(pb, q, k, k, o, cu_q=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="dtype"):
        window.WindowProblem(1, 2, 1, 64, 4, 6, dtype=torch.float32).params()
    with pytest.raises(ValueError, match="takes"):
        window.WindowBuffers(window.WindowProblem(1, 2, 3, 64, 4, 6), device="cpu")
    cache = window.PagedCache(3, 2, 64, device="cpu")
    table, lens = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    new = t(1, 4, 2, 64)
    for args, kw in (((t(1, 4, 1, 64), t(1, 4, 1, 64), table, lens), {}), ((new, t(1, 3, 2, 64), table, lens), {}),
                     ((new, new, table.long(), lens), {}), ((new, new, table, lens[:0]), {}), ((new, new, table[0], lens), {}),
                     ((t(2, 4, 2, 64), t(2, 4, 2, 64), table, lens), {}), ((new.float(), new.float(), table, lens), {}),
                     ((new[0], new[0], table, lens), dict(cu=torch.zeros(3, dtype=torch.int32)))):
        with pytest.raises(ValueError):
            cache.append(*args, **kw)
    with pytest.raises(ValueError, match="on a GPU"):
        cache.append(new, new, table, lens)
    with pytest.raises(ValueError, match="on a GPU"):
        cache.attend(t(1, 4, 4, 64), table, lens)
    with pytest.raises(ValueError):
        window.PagedCache.of(cache.k.float(), cache.v, cache.k_scale, cache.v_scale)
    assert cache.workspace_bytes(1, 4, 1, 2) > 0 and cache.workspace_bytes(1, 3, 1, 2) == 0


def test_the_binding_checks_workspaces_and_dimensions():
    from paper_2505_13389_amd.autograd import window_attention
    pb = window.WindowProblem(1, 2, 1, 64, 4, 6)
    q, k = torch.zeros(1, 4, 2, 64, dtype=BF), torch.zeros(1, 6, 1, 64, dtype=BF)
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 20, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="contiguous"):
            window.vsa_window_forward(pb, q, k, k, q.clone(), workspace=ws)
    for bad in ((q[0], k, k), (q, k[0], k), (q, k, k[0]), (q[0, 0], k[0, 0], k[0, 0])):
        with pytest.raises(ValueError):
            window_attention(*bad)
    # strides of dimensions with one entry say nothing
    odd = torch.zeros(6 * 64, dtype=BF).as_strided((1, 6, 1, 64), (3, 64, 1, 1))
    s = window._strides(odd, "k")
    assert (s.batch, s.token, s.head) == (0, 64, 0)


def test_leaves_that_another_graph_holds_are_refused(monkeypatch):
    """What window_attention checks while it is captured."""
    from paper_2505_13389_amd import autograd

    class Stream:
        cuda_stream = 5
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream)
    q, k = torch.zeros(3, requires_grad=True), torch.zeros(3, requires_grad=True)
    plain = torch.zeros(3)
    nodes = autograd._refuse_held_leaves(q, k, plain, torch.zeros(3, requires_grad=True) * 2)  # (not a leaf)
    assert len(nodes) == 2
    alive = q * 2  # of the same capture: marked with its stream
    assert len(autograd._refuse_held_leaves(q, k, plain)) == 2
    del alive, nodes
    eager = k.sin()
    with pytest.raises(RuntimeError, match="another autograd graph"):
        autograd._refuse_held_leaves(q, k)
    with torch.no_grad():
        assert autograd._refuse_held_leaves(q, k) == []
    del eager
    assert len(autograd._refuse_held_leaves(q, k)) == 2
    Stream.cuda_stream = 6
    held = k * 1
    with pytest.raises(RuntimeError):
        autograd._refuse_held_leaves(k)
    del held
