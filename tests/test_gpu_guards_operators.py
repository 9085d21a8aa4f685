"""Memory-safety evidence for the model call's operators: every output, the cache and each workspace lie between guard
regions, are poison-filled before the call, and every call is run twice and must repeat."""
import pytest
import torch

pytestmark = pytest.mark.gpu
GUARD = 64  # elements on each side


def guarded(shape, dtype, poison):
    n = 1
    for x in shape:
        n *= x
    buf = torch.full((n + 2 * GUARD,), poison, dtype=dtype, device="cuda")
    buf[:GUARD], buf[-GUARD:] = 77, 77
    return buf, buf[GUARD:GUARD + n].view(shape)


def intact(buf):
    return bool((buf[:GUARD] == 77).all() and (buf[-GUARD:] == 77).all())


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("S,N,Hq,Hkv,D,page,lens,live", [
    (1, 1, 4, 2, 64, 16, [37], None),
    (3, 23, 6, 2, 128, 32, [300, 0, 65], [23, 7, 0]),
    (2, 150, 4, 4, 64, 64, [1000, 129], [150, 149]),
    (9, 3, 8, 8, 128, 128, [2000, 1, 0, 128, 127, 129, 700, 256, 5], None),
])
def test_they_stay_inside_their_buffers_and_repeat(S, N, Hq, Hkv, D, page, lens, live, quantised):
    import paper_2411_03786_b200 as ngs
    V, M, n_alt = 1003, S * N, 7
    g = torch.Generator().manual_seed(S * N)
    w = (torch.randn(V, 64, generator=g) / 8).bfloat16().cuda()
    ctx = ngs.SpecContext(w, w)
    lib, h, P = ctx._lib, ctx._h, lambda t: t.data_ptr()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    per = -(-(max(lens) + N) // page)
    table = torch.randperm(S * per, generator=g).int().view(S, per).cuda()
    first = torch.randn(S, max(lens) + N, 2 * Hkv, D, generator=g).bfloat16().cuda()
    t = torch.randn(S, N, Hq + 2 * Hkv, D, generator=g).bfloat16().cuda()
    q, k, v = t.split([Hq, Hkv, Hkv], 2)
    rope = ngs.Rope((10000.0 ** (-torch.arange(0, 64, 2) / 64)).float().cuda())
    pos, n, nn = i32(list(range(S * N))).view(S, N), i32(lens), None if live is None else i32(live)
    parent = i32([[j - 1 if j % 4 else -1 for j in range(N)]] * S)
    hidden, tok = torch.randn(M, 64, generator=g).bfloat16().cuda(), i32([j % V for j in range(M)])
    results = []
    for _ in range(2):
        bufs = {}

        def out(name, shape, dtype=torch.bfloat16, poison=None):
            poison = poison if poison is not None else (-(1 << 30) if dtype is torch.int32 else 0x7F if dtype is torch.uint8 else float("nan"))
            bufs[name] = guarded(shape, dtype, poison)
            return bufs[name][1]
        pool = (S * per, Hkv, page, D)
        code = torch.uint8 if quantised else torch.bfloat16
        exps = [out(x, pool[:3], torch.uint8, 255) for x in ("k_exp", "v_exp")] if quantised else [None, None]
        cache = ngs.KVCache(out("cache_k", pool, code), out("cache_v", pool, code), table, *exps)
        ctx.cache_write(cache, first[:, :, :Hkv], first[:, :, Hkv:], i32([0] * S), count=n, rope=rope)
        ctx.cache_write(cache, k, v, n, nodes=i32([[j if j % 3 else -1 for j in range(N)]] * S), rope=rope)
        ctx.cache_read(cache, i32([0] * S), max(lens) + 1, count=n, out=(out("read_k", (S, max(lens) + 1, Hkv, D)), out("read_v", (S, max(lens) + 1, Hkv, D))))
        ctx.rope_rows(rope, q, k, pos, out=(out("rope_q", q.shape), out("rope_k", k.shape)))
        mask, depth = out("mask", (S, N, (N + 31) // 32), torch.int32), out("depth", (S, N), torch.int32)
        assert lib.spec_tree_mask(h, P(parent), S, N, None if nn is None else P(nn), P(mask), P(depth), None) == 0
        need = lib.spec_tree_attention_bytes(h, cache._ref, S, N, Hq)
        ctx.tree_attention(cache, q, k, v, mask, n, n_nodes=nn, out=(out("attention", q.shape), out("lse", (S, N, Hq), torch.float32)), work=out("work", (need,), torch.uint8))
        ctx.score_tokens(hidden, tok, n_alt=n_alt, work=out("score_work", (lib.spec_score_bytes(h, M, n_alt),), torch.uint8),
                         out=(out("logp", (M,), torch.float32), out("entropy", (M,), torch.float32), out("ids", (M, n_alt), torch.int32), out("alt", (M, n_alt), torch.float32)))
        torch.cuda.synchronize()
        assert ctx.get_status() == 0
        for name, (buf, _) in bufs.items():
            assert intact(buf), f"{name}: guard region overwritten"
        for name in ("read_k", "read_v", "rope_q", "rope_k", "attention", "lse", "logp", "entropy", "alt"):
            assert not bufs[name][1].isnan().any(), f"{name}: element left unwritten"
        for name in ("mask", "depth", "ids"):
            assert not (bufs[name][1] == -(1 << 30)).any(), f"{name}: element left unwritten"
        results.append({x: b[1].clone() for x, b in bufs.items() if "work" not in x})
    for name in results[0]:
        a, b = (r[name] for r in results)
        assert torch.equal(a.nan_to_num() if a.is_floating_point() else a, b.nan_to_num() if b.is_floating_point() else b), f"{name}: two identical calls disagree"
    ctx.close()
