"""Memory-safety evidence for the 4-bit cache, its attention, its pages and rotary axes: every output, the cache, the pool's table and counts
and each workspace lie between guard regions, are poison-filled before the call, and every call is run twice and must repeat."""
import pytest
import torch

from test_gpu_guards_operators import guarded, intact

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S,N,Hq,Hkv,D,page,lens,live", [
    (1, 1, 4, 2, 64, 16, [37], None),
    (3, 3, 6, 2, 128, 32, [300, 0, 65], [3, 2, 0]),
    (3, 23, 6, 2, 128, 32, [300, 0, 65], [23, 7, 0]),
    (2, 150, 4, 4, 64, 64, [1000, 129], [150, 149]),
    (9, 2, 8, 1, 128, 128, [2000, 1, 0, 128, 127, 129, 700, 256, 5], None),
    (9, 4, 8, 8, 64, 16, [2000, 1, 0, 128, 127, 129, 700, 256, 5], None),
])
def test_they_stay_inside_their_buffers_and_repeat(S, N, Hq, Hkv, D, page, lens, live):
    import paper_2411_03786_b200 as ngs
    g = torch.Generator().manual_seed(S * N)
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    ctx = ngs.SpecContext(w, w)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    per = -(-(max(lens) + N) // page)
    n_pages = S * per + 2
    first = torch.randn(S, max(lens) + N, 2 * Hkv, D, generator=g).bfloat16().cuda()
    t = torch.randn(S, N, Hq + 2 * Hkv, D, generator=g).bfloat16().cuda()
    q, k, v = t.split([Hq, Hkv, Hkv], 2)
    rope = ngs.Rope((10000.0 ** (-torch.arange(0, 64, 2) / 64)).float().cuda(), axis=(torch.arange(32) % 3).to(torch.uint8).cuda())
    pos, pos_first = (torch.randint(0, 5000, (3, S, m), generator=g).int().cuda() for m in (N, max(lens) + N))
    n, nn, zero = i32(lens), None if live is None else i32(live), i32([0] * S)
    mask = ctx.tree_mask(i32([[j - 1 if j % 4 else -1 for j in range(N)]] * S))[0]
    results = []
    for _ in range(2):
        bufs = {}

        def out(name, shape, dtype=torch.bfloat16, poison=None):
            poison = poison if poison is not None else (-(1 << 30) if dtype is torch.int32 else 0x7F if dtype is torch.uint8 else float("nan"))
            bufs[name] = guarded(shape, dtype, poison)
            return bufs[name][1]
        shape = (n_pages, Hkv, page)
        table = out("table", (S, per), torch.int32, -1)
        caches = [ngs.KVCache(out(f"k{i}", (*shape, D // 2), torch.uint8), out(f"v{i}", (*shape, D // 2), torch.uint8), table,
                              k_scale=out(f"k_scale{i}", (*shape, D // 16), torch.uint8, 255), v_scale=out(f"v_scale{i}", (*shape, D // 16), torch.uint8, 255)) for i in range(2)]
        pool = ngs.PagePool(caches, out("refs", (n_pages,), torch.int32, 0))
        work = out("page_work", (ctx._lib.spec_pages_bytes(None, pool._ref),), torch.uint8)
        ctx.pages_reserve(pool, zero, n, out=out("ok", (S,), torch.int32), work=work)
        ctx.cache_write(caches[0], first[:, :, :Hkv], first[:, :, Hkv:], zero, count=n, rope=rope, pos=pos_first)
        ctx.cache_write(caches[1], first[:, :, :Hkv], first[:, :, Hkv:], zero, count=n)
        ctx.pages_reserve(pool, n, i32([N] * S), out=out("ok2", (S,), torch.int32), work=work)
        ctx.cache_write(caches[0], k, v, n, nodes=i32([[j if j % 3 else -1 for j in range(N)]] * S))
        ctx.pages_assign(pool, i32([(s + 1) % S for s in range(S)]), torch.roll(n, -1))
        ctx.pages_assign(pool, i32([(s - 1) % S for s in range(S)]), n)
        ctx.pages_compact(pool, out=out("live", (1,), torch.int32), work=work)
        ctx.cache_read(caches[0], zero, max(lens) + 1, count=n, out=(out("read_k", (S, max(lens) + 1, Hkv, D)), out("read_v", (S, max(lens) + 1, Hkv, D))))
        ctx.rope_rows(rope, q, k, pos, out=(out("rope_q", q.shape), out("rope_k", k.shape)))
        need = ctx._lib.spec_tree_attention_bytes(ctx._h, caches[1]._ref, S, N, Hq)
        ctx.tree_attention(caches[1], q, k, v, mask, n, n_nodes=nn, out=(out("attention", q.shape), out("lse", (S, N, Hq), torch.float32)), work=out("work", (need,), torch.uint8))
        torch.cuda.synchronize()
        assert ctx.get_status() == 0
        for name, (buf, _) in bufs.items():
            assert intact(buf), f"{name}: guard region overwritten"
        for name in ("read_k", "read_v", "rope_q", "rope_k", "attention", "lse"):
            assert not bufs[name][1].isnan().any(), f"{name}: element left unwritten"
        assert bufs["ok"][1].eq(1).all() and bufs["ok2"][1].eq(1).all() and bufs["live"][1].item() == sum(-(-x // page) for x in lens)
        results.append({x: b[1].clone() for x, b in bufs.items() if "work" not in x})
    for name in results[0]:
        a, b = (r[name] for r in results)
        assert torch.equal(a.nan_to_num() if a.is_floating_point() else a, b.nan_to_num() if b.is_floating_point() else b), f"{name}: two identical calls disagree"
    ctx.close()


@pytest.mark.parametrize("N", [1, 40])
def test_an_expired_wait_ends_the_call(N):
    """Kernels that start as if a wait had expired return, say so, and leave the context usable."""
    import paper_2411_03786_b200 as ngs
    import e2m1_util as e4
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    ctx = ngs.SpecContext(w, w)
    cache, _, _ = e4.make_cache(2, 300, 2, 128, 16, 1)
    t = torch.randn(2, N, 8, 128).bfloat16().cuda()
    mask = ctx.tree_mask(torch.full((2, N), -1, dtype=torch.int32, device="cuda"))[0]
    lens = torch.tensor([300, 17], dtype=torch.int32).cuda()
    run = lambda: ctx.tree_attention(cache, t[:, :, :4], t[:, :, 4:6], t[:, :, 6:], mask, lens)[0]
    want = run()
    ctx.debug_wait_limit(0)
    run()
    assert ctx.get_status() == (0 if N == 1 else ngs.STATUS_TIMEOUT)  # (few rows: that form waits for nothing that could be lost)
    ctx.debug_wait_limit()
    assert torch.equal(run(), want) and ctx.get_status() == 0
    ctx.close()
