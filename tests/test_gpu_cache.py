"""The 8-bit cache: appending and attention over it, against their definitions in 64 bits (window_ref.py)."""
import pytest
import torch

import window_ref as ref
from paper_2505_13389_amd import window

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def filled(seed, pages, Hkv, d):
    """A pool of arbitrary values and scales, every byte a number."""
    k = (randn(seed, pages, Hkv, 64, d) * 60).clamp(-440, 440).to(torch.float8_e4m3fn)
    v = (randn(seed + 1, pages, Hkv, d, 64) * 60).clamp(-440, 440).to(torch.float8_e4m3fn)
    scale = lambda s: torch.exp2(torch.randint(-8, -3, (pages, Hkv), generator=torch.Generator().manual_seed(s)).float())
    return k, v, scale(seed + 2), scale(seed + 3)


def table_of(seed, lens, pages, columns, dtype=torch.int32):
    """Pages in no order; entries behind a sequence are not page numbers."""
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((len(lens), columns), -7, dtype=dtype)
    for b, n in enumerate(lens):
        for i in range((n + 63) // 64):
            table[b, i] = order.pop()
    return table


def cache_on_gpu(k, v, ks, vs):
    return window.PagedCache.of(k.cuda(), v.cuda(), ks.cuda(), vs.cuda())


def same_bits(cache, k8, v8, ks, vs):
    for n, got, want in (("k", cache.k, k8), ("v", cache.v, v8)):
        got = got.float().cpu().double()
        bad = ~((got == want) | (got.isnan() & want.isnan()))
        assert not bad.any(), f"{n}: {int(bad.sum())} values differ, first at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]}"
    assert torch.equal(cache.k_scale.cpu().double(), ks) and torch.equal(cache.v_scale.cpu().double(), vs)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("Hkv,d", [(1, 64), (3, 128)])
def test_append_packed(dtype, Hkv, d):
    """Beginnings and ends inside pages, whole pages, nothing, scales that grow and that stay."""
    before, new = [0, 5, 64, 63, 100, 130, 60, 17], [64, 3, 200, 1, 0, 70, 4, 1]
    lens = [a + b for a, b in zip(before, new)]
    pool = filled(1, 24, Hkv, d)
    table = table_of(2, lens, 24, 5)
    k = (randn(5, sum(new), Hkv, d) * torch.exp2(torch.randint(-6, 6, (sum(new), 1, 1), generator=torch.Generator().manual_seed(6)).float())).to(dtype)
    v = randn(7, sum(new), Hkv, d).to(dtype)
    cache = cache_on_gpu(*pool)
    cu = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    junk = torch.full((2, Hkv, d), float("nan"), dtype=dtype, device="cuda")  # behind the last sequence
    cache.append(torch.cat([k.cuda(), junk]), torch.cat([v.cuda(), junk]), table.cuda(), torch.tensor(before, dtype=torch.int32, device="cuda"), cu=cu)
    want = [t.double() for t in pool]
    at = 0
    for b, n in enumerate(new):
        ref.append(*want, k[at:at + n], v[at:at + n], [int(x) for x in table[b]], before[b])
        at += n
    same_bits(cache, *want)


def test_append_token_by_token_and_special_values():
    """A page filled one token at a time, through zeros, tiny and huge values, infinities and NaN; strided, dense tensors."""
    Hkv, d = 2, 64
    pool = filled(3, 4, Hkv, d)
    table = torch.tensor([[2, 0], [3, 1]], dtype=torch.int32)
    cache, want = cache_on_gpu(*pool), [t.double() for t in pool]
    for i in range(70):
        k, v = randn(100 + i, 2, 1, Hkv, d).to(BF), randn(200 + i, 2, 1, Hkv, d).to(BF)
        if i < 3:
            k.zero_()
        if i % 7 == 3:
            k *= 2.0 ** (i - 20)
        if i == 30:
            v[0, 0, 0, 5] = float("inf")
            v[1, 0, 1, 6] = float("nan")
        if i == 40:
            v[0] = 3e38
        if i == 66:
            k[:] = 1e-38
        both = torch.cat([k, v], 3)
        kk, vv = both.cuda()[..., :d], both.cuda()[..., d:]
        cache.append(kk, vv, table.cuda(), torch.full((2,), i, dtype=torch.int32, device="cuda"))
        for b in range(2):
            ref.append(*want, k[b], v[b], table[b].tolist(), i)
    same_bits(cache, *want)


def test_append_drops_what_has_no_page():
    Hkv, d = 2, 128
    pool = filled(4, 3, Hkv, d)
    table = torch.tensor([[1, -1, 900, 2]], dtype=torch.int32)
    k, v = randn(1, 1, 300, Hkv, d).to(BF), randn(2, 1, 300, Hkv, d).to(BF)  # 300 tokens behind 10: the last 54 have no entry
    cache, want = cache_on_gpu(*pool), [t.double() for t in pool]
    cache.append(k.cuda(), v.cuda(), table.cuda(), torch.tensor([10], dtype=torch.int32, device="cuda"))
    ref.append(*want, k[0], v[0], [1, None, None, 2], 10)
    same_bits(cache, *want)


MASKS = {"all_before": (-1, 0, 0, 1), "window": (100, 0, 4, 1), "frames": (1, 0, 1, 70), "sinks_only_far": (0, 0, 65, 1), "ahead": (30, 9, 0, 1)}


def attend_case(seed, lens, new, H, Hkv, d, dtype, mask, columns, hole=None, dirty=True):
    pages = sum((n + 63) // 64 for n in lens) + 2
    k8, v8, ks, vs = filled(seed, pages, Hkv, d)
    table = table_of(seed, lens, pages, columns)
    if hole is not None:
        table[hole] = pages + 5
    if dirty:  # slots behind the last token: NaN
        for b, n in enumerate(lens):
            if n % 64:
                page = int(table[b, n // 64])
                if 0 <= page < pages:
                    k8.view(torch.uint8)[page, :, n % 64:] = 0x7F
                    v8.view(torch.uint8)[page, :, :, n % 64:] = 0xFF
    # logits of order one: keys are of order 60 * 2^-5
    q = (randn(seed + 9, sum(new), H, d) * (0.5 if dtype == BF else 0.25)).to(dtype)
    left, right, sinks, unit = mask
    cache = cache_on_gpu(k8, v8, ks, vs)
    cu = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    lens_d = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = torch.full((q.shape[0] + 2, H, d), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((H, q.shape[0] + 2), 7.0, device="cuda")
    qd = torch.cat([q.cuda(), torch.full((2, H, d), float("nan"), dtype=dtype, device="cuda")])
    got = cache.attend(qd, table.cuda(), lens_d, cu=cu, max_q=max(new), left=left, right=right, sinks=sinks, unit=unit, out=out, lse=lse)
    assert got is out and (out[-2:] == 7.0).all() and (lse[:, -2:] == 7.0).all()
    at = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        ids = [int(x) if 0 <= x < pages else None for x in table[b]]
        k, v, there = ref.cached(k8, v8, ks, vs, ids, n)
        want = ref.attention(q[at:at + m], k, v, ref.visible(m, n, *mask) & there[None], out_type=dtype)
        ref.check(out[at:at + m], want["out"], f"out of sequence {b}: {m} queries, {n} tokens")
        ref.check(lse[:, at:at + m], want["lse"], f"lse of sequence {b}")
        at += m


@pytest.mark.parametrize("mask", MASKS.values(), ids=MASKS.keys())
@pytest.mark.parametrize("H,Hkv,d,dtype", [(4, 1, 128, BF), (3, 3, 64, FP), (20, 1, 64, BF), (16, 2, 128, FP)])
def test_single_tokens(mask, H, Hkv, d, dtype):
    attend_case(1, [1, 64, 65, 700, 1999], [1, 1, 1, 1, 1], H, Hkv, d, dtype, mask, 40)


@pytest.mark.parametrize("mask", MASKS.values(), ids=MASKS.keys())
@pytest.mark.parametrize("H,Hkv,d,dtype", [(4, 2, 128, BF), (3, 1, 64, FP)])
def test_few_queries(mask, H, Hkv, d, dtype):
    """Several query tiles, sequences without queries, more queries than tokens."""
    attend_case(2, [40, 128, 0, 900, 333, 5], [7, 19, 0, 33, 0, 9], H, Hkv, d, dtype, mask, 16)


@pytest.mark.parametrize("mask", MASKS.values(), ids=MASKS.keys())
@pytest.mark.parametrize("H,Hkv,d,dtype", [(4, 2, 128, BF), (2, 2, 64, BF), (6, 2, 128, FP), (3, 1, 64, FP)])
def test_chunks(mask, H, Hkv, d, dtype):
    attend_case(3, [150, 400, 90, 64, 777], [150, 131, 200, 64, 1], H, Hkv, d, dtype, mask, 16)


def test_chunks_with_a_wavefront_a_block():
    attend_case(4, [300] * 9, [200] * 9, 16, 16, 128, BF, (100, 0, 4, 1), 6)


@pytest.mark.parametrize("new", [[1, 1], [150, 170]])
def test_entries_that_name_no_page_hide_their_tokens(new):
    attend_case(5, [500, 640], new, 4, 2, 128, BF, (-1, 0, 0, 1), 12, hole=(0, 3))


def test_many_parts():
    """A long sequence whose pages are split over many workgroups, beside a short one."""
    attend_case(6, [30011, 70], [1, 1], 8, 1, 64, BF, (-1, 0, 0, 1), 512)


@pytest.mark.parametrize("new", [[1, 0, 1], [40, 1, 60], [260, 0, 140]])
@pytest.mark.parametrize("d", [64, 128])
def test_short_calls_on_a_long_cache(new, d):
    """Walks in parts, whichever kernel has them: single tokens, few queries, a chunk."""
    attend_case(7, [4001, 64, 2900], new, 4, 2, d, BF, (-1, 0, 0, 1), 80)
    attend_case(8, [4001, 64, 2900], new, 4, 2, d, FP, (2000, 0, 70, 1), 80)


@pytest.mark.parametrize("columns", [4, 16, 17, 32, 33])
def test_short_tables(columns):
    """Caches that one workgroup walks alone, and the first that it does not."""
    lens = [min(n, 64 * columns) for n in (1, 200, 1024, 1025, 2048, 2049)]
    attend_case(9, lens, [1, 1, 3, 1, 0, 2], 4, 2, 128, BF, (-1, 0, 0, 1), columns)
    attend_case(10, lens, [1, 1, 3, 1, 0, 2], 6, 2, 64, FP, (70, 0, 3, 1), columns)


def test_more_sequences_than_lanes():
    """130 sequences, some empty or without queries, tables of many and of few columns."""
    lens = [i * 37 % 301 for i in range(130)]
    new = [min(i % 3, n) for i, n in enumerate(lens)]
    for columns in (5, 40):
        attend_case(11, lens, new, 4, 2, 64, BF, (100, 0, 4, 1), columns)
    attend_case(12, lens, [130 if i == 77 else x for i, x in enumerate(new)], 2, 2, 64, BF, (100, 0, 4, 1), 40)


def test_parts_of_more_than_64_pages_a_wavefront():
    """Long sequences that fill the chip by themselves; their pages repeat, so that the pool stays small."""
    B, H, Hkv, d, n = 40, 8, 8, 64, 70399
    k8, v8, ks, vs = filled(13, 50, Hkv, d)
    table = torch.randint(0, 50, (B, 1101), generator=torch.Generator().manual_seed(14), dtype=torch.int32)
    q = (randn(15, B, 1, H, d) * 0.5).to(BF)
    lens = torch.full((B,), n, dtype=torch.int32)
    got = cache_on_gpu(k8, v8, ks, vs).attend(q.cuda(), table.cuda(), lens.cuda())
    for b in (0, 23, 39):
        k, v, _ = ref.cached(k8, v8, ks, vs, table[b].tolist(), n)
        ref.check(got[b], ref.attention(q[b], k, v, torch.ones(1, n, dtype=torch.bool))["out"], f"sequence {b}")


def test_lengths_that_lie_stay_in_bounds():
    """Lengths below zero or beyond the table are taken as its ends; pages of no table stay as they were."""
    Hkv, d, columns = 2, 64, 3
    pool = filled(21, 12, Hkv, d)
    table = torch.tensor([[1, 3, 5], [7, 9, 11], [0, 2, 4]], dtype=torch.int32, device="cuda")
    wrong = torch.tensor([-9, 2 ** 31 - 1, 40], dtype=torch.int32, device="cuda")
    right = torch.tensor([0, 64 * columns, 40], dtype=torch.int32, device="cuda")
    for n in (1, 150):
        k, v, q = (randn(22 + i, 3, n, h, d).to(BF).cuda() for i, h in enumerate((Hkv, Hkv, 4)))
        a, b = cache_on_gpu(*pool), cache_on_gpu(*pool)
        a.append(k, v, table, wrong)
        b.append(k, v, table, right)
        for x, y in ((a.k.view(torch.uint8), b.k.view(torch.uint8)), (a.v.view(torch.uint8), b.v.view(torch.uint8)), (a.k_scale, b.k_scale)):
            assert torch.equal(x, y)
        for t in (a.k, a.v):
            untouched = [6, 7, 8, 9, 10, 11]  # of no table, or behind the second sequence's last page
            assert torch.equal(t[untouched].view(torch.uint8).cpu(), (pool[0] if t is a.k else pool[1])[untouched].view(torch.uint8))
        assert torch.equal(a.attend(q, table, wrong), b.attend(q, table, right))


def test_two_graphs_share_a_workspace():
    """Single tokens and a chunk, captured over one workspace and replayed in turn."""
    Hkv, d = 2, 128
    cache = cache_on_gpu(*filled(25, 60, Hkv, d))
    table = torch.randperm(60, generator=torch.Generator().manual_seed(26))[:40][None].int().cuda()
    lens = torch.tensor([2500], dtype=torch.int32, device="cuda")
    work = torch.empty(max(cache.workspace_bytes(1, 8, n, 40) for n in (1, 200)), dtype=torch.uint8, device="cuda")
    steps = []
    for n in (1, 200):
        q = (randn(27 + n, 1, n, 8, d) * 0.5).to(BF).cuda()
        want, out = cache.attend(q, table, lens, workspace=work).clone(), torch.zeros_like(q)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.attend(q, table, lens, out=out, workspace=work)
        steps.append((graph, out, want, q))
    for _ in range(4):
        work.fill_(0xFF)
        for graph, out, *_ in steps:
            out.fill_(3.0)
            graph.replay()
        torch.cuda.synchronize()
        for _, out, want, _ in steps:
            assert torch.equal(out, want)


def test_two_attentions_at_once():
    """Two streams on one cache, each with a workspace of its own."""
    Hkv, d, n = 2, 128, 3000
    cache = cache_on_gpu(*filled(16, 100, Hkv, d))
    tables = [torch.randperm(100, generator=torch.Generator().manual_seed(i))[:48][None].int().cuda() for i in range(2)]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    qs = [(randn(17 + i, 1, m, 8, d) * 0.5).to(BF).cuda() for i, m in enumerate((1, 300))]
    wants = [cache.attend(q, t, lens) for q, t in zip(qs, tables)]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in qs], [[], []]
    for _ in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs[i].append(cache.attend(qs[i], tables[i], lens))
    torch.cuda.synchronize()
    for want, got in zip(wants, outs):
        assert all(torch.equal(want, t) for t in got)


def test_timing_records_name_the_kernels():
    """The per-call timing of the other entry points covers these."""
    import ctypes as C
    from paper_2505_13389_amd import vsa
    cache = cache_on_gpu(*filled(18, 4, 2, 64))
    table, lens = torch.tensor([[0, 2]], dtype=torch.int32, device="cuda"), torch.tensor([60], dtype=torch.int32, device="cuda")
    k, q = randn(19, 1, 5, 2, 64).to(BF).cuda(), randn(20, 1, 5, 2, 64).to(BF).cuda()
    lib = vsa.lib()
    assert lib.vsa_profile_begin(8) == 0
    cache.append(k, k, table, lens)
    cache.attend(q, table, lens + 5)
    torch.cuda.synchronize()
    names = [lib.vsa_profile_name(i) for i in range(lib.vsa_profile_count())]
    times = [lib.vsa_profile_ms(i) for i in range(lib.vsa_profile_count())]
    assert lib.vsa_profile_end() == 0
    names = [n.decode() if isinstance(n, bytes) else n for n in names]
    assert len(names) == 2 and all("cache" in n for n in names) and all(0 < t < 1000 for t in times), (names, times)


def test_pool_past_32_bits():
    """Pages behind 2^32 bytes of the pool, read and written."""
    Hkv, d, pages, last = 8, 128, 70000, 69990
    cache = window.PagedCache(pages, Hkv, d)
    table = torch.tensor([[last, 3, last - 1]], dtype=torch.int32, device="cuda")
    k, v, q = randn(1, 1, 150, Hkv, d).to(BF), randn(2, 1, 150, Hkv, d).to(BF), randn(3, 1, 1, Hkv, d).to(BF)
    cache.append(k.cuda(), v.cuda(), table, torch.zeros(1, dtype=torch.int32, device="cuda"))
    lens = torch.tensor([150], dtype=torch.int32, device="cuda")
    pick = [last, 3, last - 1]
    k8, v8, ks, vs = (t[pick].cpu() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale))
    want = [torch.zeros(3, Hkv, 64, d, dtype=torch.float64), torch.zeros(3, Hkv, d, 64, dtype=torch.float64),
            torch.ones(3, Hkv, dtype=torch.float64), torch.ones(3, Hkv, dtype=torch.float64)]
    ref.append(*want, k[0], v[0], [0, 1, 2], 0)
    assert torch.equal(k8.double(), want[0]) and torch.equal(v8.double(), want[1]) and torch.equal(ks.double(), want[2])
    kk, vv, _ = ref.cached(k8, v8, ks, vs, [0, 1, 2], 150)
    for n in (1, 140):
        qn = randn(4, 1, n, Hkv, d).to(BF)
        got = cache.attend(qn.cuda(), table, lens)
        ref.check(got[0], ref.attention(qn[0], kk, vv, ref.visible(n, 150, -1, 0, 0, 1))["out"], "out")


def test_append_and_attend_captured_and_replayed():
    """A step of generation, append then attend, in a graph whose inputs, lengths among them, change between replays."""
    B, H, Hkv, d = 2, 4, 2, 128
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros(B, 1, n, d, dtype=BF, device="cuda") for n in (H, Hkv, Hkv))
    eager, graphed = window.PagedCache(8, Hkv, d), window.PagedCache(8, Hkv, d)
    out = torch.zeros_like(q)

    def step(cache, to):
        cache.append(k, v, table, lens)
        lens.add_(1)
        cache.attend(q, table, lens, left=90, sinks=2, out=to)
        lens.sub_(1)
    step(graphed, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed, out)
    for i in range(130):
        for j, t in enumerate((q, k, v)):
            t.copy_(randn(1000 + 3 * i + j, *t.shape))
        lens.fill_(i)
        want = torch.zeros_like(q)
        step(eager, want)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
    assert torch.equal(eager.k.view(torch.uint8), graphed.k.view(torch.uint8)) and torch.equal(eager.v_scale, graphed.v_scale)


def test_generation_follows_the_training_mask():
    """A clip attended whole against the same frames one by one through the cache: equal up to the cache's 8 bits."""
    frames, unit, H, Hkv, d, left, sinks = 6, 50, 4, 2, 64, 2, 1
    n = frames * unit
    q, k, v = (randn(i, 1, n, h, d).to(BF).cuda() for i, h in enumerate((H, Hkv, Hkv)))
    cache = window.PagedCache(8, Hkv, d)
    table = torch.arange(5, dtype=torch.int32, device="cuda")[None] + 1
    outs = []
    for f in range(frames):
        new = slice(f * unit, (f + 1) * unit)
        cache.append(k[:, new], v[:, new], table, torch.tensor([f * unit], dtype=torch.int32, device="cuda"))
        outs.append(cache.attend(q[:, new], table, torch.tensor([(f + 1) * unit], dtype=torch.int32, device="cuda"), left=left, sinks=sinks, unit=unit))
    # the whole clip over the keys and values that the cache stands for (bf16 holds e4m3 times a power of two exactly)
    kk, vv, _ = ref.cached(cache.k.cpu(), cache.v.cpu(), cache.k_scale.cpu(), cache.v_scale.cpu(), [1, 2, 3, 4, 5], n)
    pb = window.WindowProblem(1, H, Hkv, d, n, n, left, 0, sinks, unit)
    buf = window.WindowBuffers(pb, backward=False)
    buf.forward(q, kk.to(BF).cuda()[None], vv.to(BF).cuda()[None])
    want = ref.attention(q[0].cpu(), kk, vv, ref.visible(n, n, left, 0, sinks, unit))["out"]
    ref.check(buf.out[0], want, "whole clip")
    # (a frame's page scales may have grown after it was read: its values then moved by half a step of the 8 bits at most, if at all)
    value, off = want
    ref.check(torch.cat(outs, 1)[0], (value, off + 2.0 ** -4 * value.abs() + 2.0 ** -4), "frame by frame")
