"""The calls on 8-bit keys and values as a serving program makes them: a context's projection is rotated, clustered and quantized,
then sequences grow token by token, each step appending, selecting and attending."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from paper_2411_09688_amd import binding as sq
from test_gpu_q8_rows import cu, table

pytestmark = pytest.mark.gpu
SCALE = float(np.float32(1 / np.sqrt(128)))
F16, F32, I32 = torch.float16, torch.float32, torch.int32
EPS = 2.0 ** -20




@pytest.mark.parametrize("one_set,B,H,G,page", [(False, 2, 2, 3, 16), (True, 3, 2, 4, 32), (False, 1, 3, 1, 64)])
def test_a_context_and_the_sequences_behind_it(one_set, B, H, G, page):
    rng = np.random.default_rng(B * 10 + G)
    L, C_, steps, prompt = 700, 24, 20, 37
    cs = table(L + 100, 128)
    w = [(1 + 0.1 * rng.standard_normal(128)).astype(np.float16) for _ in range(2)]
    rot = sq.make_rotary(cu(cs), False, cu(w[0]), cu(w[1]), eps=EPS)
    e = lambda *s, dtype=F16: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731

    # the context: rotated, clustered, quantized through the order of the clusters
    x = cu((rng.standard_normal((L, 2 * H, 128)) + 2 * rng.standard_normal((C_, 2 * H, 128))[rng.integers(0, C_, L)]).astype(np.float16))
    K, V = e(1, H, L, 128), e(1, H, L, 128)
    one = sq.make_shape(1, H, 1, 1, L, 0, 1.0)
    sq.sq_head_norm_rotate(one, G, rot, torch.arange(L, dtype=I32, device="cuda"), None, x[:, :H], x[:, H:], None, K, V)
    flat = sq.make_shape(1, H, L, C_, 1, 0, 1.0)
    X = e(1, H, L, 128)
    sq.sq_kmeans_normalize(flat, K, X)
    centers = X[:, :, torch.randperm(L, generator=torch.Generator().manual_seed(3))[:C_].cuda()].contiguous()
    assign, sizes, offsets, perm = e(1, H, L, dtype=I32), e(1, H, C_, dtype=I32), e(1, H, C_ + 1, dtype=I32), e(1, H, L, dtype=I32)
    ws = sq.workspace(flat, sq.SQ_CALL_KMEANS_STEP, "cuda:0")
    for _ in range(3):
        sq.sq_kmeans_step(flat, X, centers, centers, assign, sizes, offsets, perm, ws)
    Ks, Vs, cent = e(1, H, L, 128), e(1, H, L, 128), e(1, H, C_, 128)
    sq.sq_cluster_layout(flat, K, V, perm, sizes, offsets, Ks, Vs, cent)
    n = -(-L // 64)
    K8, V8, ks, vs = e(1, H, L, 128, dtype=sq.F8), e(1, H, L, 128, dtype=sq.F8), e(1, H, n, dtype=F32), e(1, H, n, dtype=F32)
    sq.sq_kv_quantize(flat, K, V, perm, K8, V8, ks, vs)
    for src, codes, scale in ((Ks, K8, ks), (Vs, V8, vs)):     # the sorted tensors' own 8-bit form
        c, s = ref.quantize(src.cpu().numpy(), None)
        assert np.array_equal(codes.view(torch.uint8).cpu().numpy(), c) and np.array_equal(scale.cpu().numpy(), s)
    value = [ref.VALUES[c.view(torch.uint8).cpu().numpy()[0]] * s.cpu().numpy()[0].repeat(64, 1)[:, :L, None] for c, s in ((K8, ks), (V8, vs))]

    # the sequences: a prompt each, then a token at a time
    width = -(-(prompt + steps) // page)
    pages = rng.permutation(B * width + 1)[:B * width].reshape(B, width).astype(np.int32)
    codes = [np.full((B * width + 1, H, page, 128), 0x7f, np.uint8) for _ in range(2)]
    scales = [np.ones((B * width + 1, H)) for _ in range(2)]
    cache = sq.make_cache(*(cu(c).view(sq.F8) for c in codes), *(cu(s.astype(np.float32)) for s in scales), cu(pages))
    sh = sq.make_shape(B, H, L, C_, G, 0, SCALE)
    one_token = sq.make_shape(B, H, L, C_, 1, 0, SCALE)
    thresh = torch.full((H,), 1.0 / L, device="cuda")
    rows = (B, H) if one_set else (B, H * G)
    logits, row_max, denom = e(B, H, G, C_, dtype=F32), e(B, H, G, dtype=F32), e(B, H, G, dtype=F32)
    mask, ranges = e(*rows, 1, dtype=I32), torch.zeros(*rows, C_, 2, dtype=I32, device="cuda")
    n_ranges, n_keys = e(*rows, dtype=I32), e(*rows, dtype=I32)
    out, lse = e(B, H * G, 1, 128), e(B, H * G, 1, dtype=F32)
    ws_mean, ws8 = sq.workspace(sh, sq.SQ_CALL_SELECT_MEAN, "cuda:0"), sq.workspace(sh, sq.SQ_CALL_ATTN_DECODE_Q8, "cuda:0")
    held = [0] * B
    for step in range(steps):
        new = [prompt - 5 * b for b in range(B)] if step == 0 else [1] * B
        T = sum(new)
        x = cu(rng.standard_normal((T, H * G + 2 * H, 128)).astype(np.float16))
        pos = np.concatenate([L + held[b] + np.arange(new[b]) for b in range(B)]).astype(np.int32)
        first = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        q = torch.full((T, H * G, 128), 9.0, dtype=F16, device="cuda")
        parts = (x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:])
        before = cu(np.asarray(held, np.int32))
        sq.sq_cache_append(one_token, G, rot, cache, before, cu(pos), *parts, q, cu(first) if step == 0 else None)
        xn = x.cpu().numpy()
        k64 = ref.norm_rotate(xn[:, H * G:H * G + H], w[1], EPS, cs, pos, False)
        for i, src in ((0, k64), (1, xn[:, H * G + H:].astype(np.float64))):
            ref.append(codes[i], scales[i], pages, held, new, first, src)
        held = [a + b for a, b in zip(held, new)]
        last = torch.from_numpy(first[1:] - 1).cuda().long()
        q1 = q[last].contiguous()                               # [B, H*G, 128]: the newest token of each sequence
        sq.sq_centroid_score(sh, q1, cent, sizes, logits, row_max, denom)
        if one_set:
            sq.sq_select_mean(sh, logits, row_max, denom, thresh, sizes, offsets, mask, ranges, n_ranges, n_keys, ws_mean)
        else:
            sq.sq_select(sh, logits, row_max, denom, thresh, sizes, offsets, mask, ranges, n_ranges, n_keys)
        sq.sq_sparse_attn_decode_q8(sh, one_set, q1, K8, V8, ks, vs, ranges, n_ranges, n_keys, cache, cu(np.asarray(held, np.int32)), out, lse, ws8)
        rg, nr = ranges.cpu().numpy().reshape(-1, C_, 2), n_ranges.cpu().numpy().reshape(-1)
        qn, on, ln = q1.cpu().numpy().astype(np.float64), out.cpu().numpy()[:, :, 0].astype(np.float64), lse.cpu().numpy()[:, :, 0]
        for b in range(B):
            t = np.arange(held[b])
            for h in range(H):
                user = [ref.VALUES[codes[i][pages[b, t // page], h, t % page]] * scales[i][pages[b, t // page], h][:, None] for i in range(2)]
                for g in range(G):
                    r = b * H + h if one_set else (b * H + h) * G + g
                    ids = np.concatenate([np.arange(s, s + c) for s, c in rg[r, :nr[r]]] + [np.zeros(0, int)]).astype(int)
                    assert len(ids) == n_keys.reshape(-1)[r].item()
                    k, v = (np.concatenate([value[i][h, ids], user[i]]) for i in range(2))
                    o, z, moved = ref.attend(qn[b, h * G + g][None], k, v, SCALE)
                    off = np.abs(on[b, h * G + g] - o[0]) - np.abs(o[0]) * 2.0 ** -11 - 2.0 ** -25
                    assert off.max() <= moved[0, 0], (step, b, h, g, off.max(), moved)
                    assert abs(ln[b, h * G + g] - z[0]) <= moved[0, 1] + abs(z[0]) * 2.0 ** -22
    for i in range(2):
        got = cache.tensors[i].view(torch.uint8).cpu().numpy()
        assert ref.same_codes(got, codes[i]).all() and np.array_equal(cache.tensors[2 + i].cpu().numpy(), scales[i].astype(np.float32))


def test_a_pool_of_more_than_4_gb():
    """Pages behind the reach of 32-bit offsets: appended to, and attended to by rows of their own and by the union."""
    H, P = 8, 64
    n = (1 << 32) // (H * P * 128) + 40
    free, _ = torch.cuda.mem_get_info()
    assert free > 3 * n * H * P * 128
    rng = np.random.default_rng(9)
    B = 8
    pages = (n - 1 - rng.permutation(B * 2)).reshape(B, 2).astype(np.int32)    # the last of the pool
    K8, V8 = (torch.zeros(n, H, P, 128, dtype=torch.uint8, device="cuda").view(sq.F8) for _ in range(2))
    ks, vs = (torch.ones(n, H, device="cuda") for _ in range(2))
    cache = sq.make_cache(K8, V8, ks, vs, cu(pages))
    new = [70 + 7 * b for b in range(B)]
    T = sum(new)
    x = [rng.standard_normal((T, H, 128)).astype(np.float16) for _ in range(2)]
    first = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    one = sq.make_shape(B, H, 1, 1, 1, 0, SCALE)
    sq.sq_cache_append(one, 1, sq.make_rotary(None), cache, torch.zeros(B, dtype=I32, device="cuda"), None, None, cu(x[0]), cu(x[1]), None, cu(first))
    held = cu(np.asarray(new, np.int32))
    q = rng.standard_normal((B, H, 128)).astype(np.float16)
    used = pages.reshape(-1)
    codes, scales = [np.zeros((B * 2, H, P, 128), np.uint8) for _ in range(2)], [np.ones((B * 2, H)) for _ in range(2)]
    local = np.arange(B * 2).reshape(B, 2)
    for i in range(2):
        ref.append(codes[i], scales[i], local, [0] * B, new, first, x[i].astype(np.float64))
        assert np.array_equal((K8, V8)[i].view(torch.uint8)[torch.from_numpy(used).cuda().long()].cpu().numpy(), codes[i])
        assert np.array_equal((ks, vs)[i][torch.from_numpy(used).cuda().long()].cpu().numpy(), scales[i].astype(np.float32))
    for L in (None, 32768, 131072):                             # 8 sequences x 8 heads x 32768 keys: the union; 131072: past the caches
        sh = sq.make_shape(B, H, L or 1, 2, 1, 0, SCALE)
        fixed = [None] * 7
        if L:
            bits = rng.integers(0, 0x7f, (2, H, L, 128), np.uint8)
            fs = torch.full((H, L // 64), 2.0 ** -7, device="cuda")
            ranges = np.zeros((B * H, 2, 2), np.int32)
            ranges[:, 0] = np.stack([rng.integers(0, L - 200, B * H), rng.integers(0, 200, B * H)], 1)
            nr = np.ones(B * H, np.int32)
            fixed = [cu(bits[0]).view(sq.F8), cu(bits[1]).view(sq.F8), fs, fs, cu(ranges), cu(nr), cu(ranges[:, 0, 1].copy())]
        out, lse = torch.empty(B, H, 1, 128, dtype=F16, device="cuda"), torch.empty(B, H, 1, device="cuda")
        ws = sq.workspace(sh, sq.SQ_CALL_ATTN_DECODE_Q8, "cuda:0")
        sq.sq_sparse_attn_decode_q8(sh, False, cu(q), *fixed, cache, held, out, lse, ws)
        for b in range(B):
            t = np.arange(new[b])
            for h in range(H):
                k, v = (ref.VALUES[codes[i][local[b, t // P], h, t % P]] * scales[i][local[b, t // P], h][:, None] for i in range(2))
                if L:
                    s, c = ranges[b * H + h, 0]
                    k, v = (np.concatenate([ref.VALUES[bits[i][h, s:s + c]] * 2.0 ** -7, y]) for i, y in ((0, k), (1, v)))
                o, z, moved = ref.attend(q[b, h][None].astype(np.float64), k, v, SCALE)
                off = np.abs(out[b, h, 0].cpu().numpy().astype(np.float64) - o[0]) - np.abs(o[0]) * 2.0 ** -11 - 2.0 ** -25
                assert off.max() <= moved[0, 0], (L, b, h)


def test_the_binding_refuses_tensors_that_do_not_fit():
    t = lambda *s, dtype=F16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    sh = sq.make_shape(2, 3, 100, 5, 4, 0, 0.1)
    K8 = t(3, 100, 128, dtype=torch.uint8).view(sq.F8)
    pool = t(5, 3, 16, 128, dtype=torch.uint8).view(sq.F8)
    cache = sq.make_cache(pool, pool.clone(), t(5, 3, dtype=F32), t(5, 3, dtype=F32), t(2, 4, dtype=I32))
    ok = dict(q=t(2, 12, 1, 128), K8=K8, V8=K8, ks=t(3, 2, dtype=F32), vs=t(3, 2, dtype=F32), ranges=t(24, 5, 2, dtype=I32),
              nr=t(24, dtype=I32), nk=t(24, dtype=I32), cache=cache, seq=t(2, dtype=I32), out=t(2, 12, 1, 128), lse=t(2, 12, 1, dtype=F32),
              ws=sq.workspace(sh, sq.SQ_CALL_ATTN_DECODE_Q8, "cuda:0"))
    call = lambda **kw: sq.sq_sparse_attn_decode_q8(sh, False, *{**ok, **kw}.values())  # noqa: E731
    call()
    for bad in (dict(q=t(2, 12, 1, 64)), dict(K8=t(3, 100, 128)), dict(ks=t(3, 3, dtype=F32)), dict(ranges=t(6, 5, 2, dtype=I32)),
                dict(lse=t(2, 12, 1)), dict(seq=torch.zeros(2, dtype=I32)), dict(out=t(2, 12, 2, 128)[:, :, :1]),
                dict(cache=sq.make_cache(pool, pool, t(5, 3, dtype=F32), t(5, 3, dtype=F32), t(1, 4, dtype=I32)))):
        with pytest.raises(ValueError):
            call(**bad)
    rot = sq.make_rotary(t(8, 64, 2, dtype=F32))
    rows = dict(q=t(2, 6, 128), k=t(2, 3, 128), v=t(2, 3, 128))
    one = sq.make_shape(2, 3, 1, 1, 1, 0, 1.0)
    app = lambda **kw: sq.sq_cache_append(one, 2, rot, cache, t(2, dtype=I32), t(2, dtype=I32), *{**rows, **kw}.values(), t(2, 6, 128))  # noqa: E731
    app()
    for bad in (dict(q=t(2, 6, 256)[:, :, ::2]), dict(k=t(2, 4, 128)), dict(v=t(3, 2, 128).transpose(0, 1)), dict(k=t(2, 3, 128, dtype=F32))):
        with pytest.raises(ValueError):
            app(**bad)
    with pytest.raises(ValueError):
        sq.make_rotary(t(8, 64, 2))
    with pytest.raises(sq.SqError):
        sq.sq_cache_append(one, 2, rot, cache, t(2, dtype=I32), t(2, dtype=I32), rows["q"], rows["k"], rows["v"], rows["q"])
    torch.cuda.synchronize()
