"""The model-side calls at the ends of the ranges that their arguments are documented for.
References are plain, in 64 bits; bounds come from the arithmetic (see model_ref.py).
"""
import math

import numpy as np
import pytest
import torch

import model_ref as ref
import paper_2412_01447_amd as pld
from gpu_helpers import d_i32, dev, say
from model_ref import U, f64
from paper_2412_01447_amd.cache import PagedCache
from test_gpu_model import E4M3, Case, bits, normal

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ log probabilities
def logprobs(z, tokens, count=None, tau=1.0, top=5):
    """(log probabilities, entropies, ids, their log probabilities), 7 or -7 where nothing was written."""
    B, n, V = z.shape
    lp, ent = torch.full((B, n), 7.0, device=dev()), torch.full((B, n), 7.0, device=dev())
    ids, tl = torch.full((B, n, top), -7, dtype=torch.int32, device=dev()), torch.full((B, n, top), 7.0, device=dev())
    need = pld.pld_token_logprobs_workspace_bytes(B, n, V, pld.PLD_F32 if z.dtype == torch.float32 else pld.PLD_BF16, top)
    ws = torch.full((need,), 0x7f, dtype=torch.uint8, device=dev())
    pld.pld_token_logprobs(z, tokens, lp, ws, count=count, temperature=tau, entropy=ent, top_ids=ids, top_logprobs=tl)
    return lp, ent, ids, tl


def close(x, y, V):
    """A lane's share of the sum, the tree over lanes and parts, the exponentials (as in test_token_logprobs)."""
    return (x - y).abs() <= (V / 64 + 96) * U + 8 * U * (y.abs() + 1)


@pytest.mark.parametrize("B,n,V,dtype", [(1, 4096, 300, "f32"), (1, 4097, 300, "f32"), (4, 2048, 32000, "bf16"),
                                         (512, 9, 3000, "f32"), (64, 65, 6000, "bf16"), (4096, 11, 70, "f32"),
                                         (2, 30000, 2049, "bf16")])
def test_more_rows_than_waves(B, n, V, dtype):
    """Several rows begin in one wave's share, sequences without rows among them."""
    say("rows", B, n, V, dtype)
    g = torch.Generator(device=dev()).manual_seed(B + n)
    z = torch.randn(B, n, V, generator=g, device=dev(), dtype=torch.float32 if dtype == "f32" else torch.bfloat16).mul_(3)
    tokens = torch.randint(0, V, (B, n), generator=g, device=dev(), dtype=torch.int32)
    for count in (None, torch.randint(-1, n + 2, (B,), generator=g, device=dev(), dtype=torch.int32)):
        lp, ent, ids, tl = logprobs(z, tokens, count)
        add = (V / 64 + 96) * U
        for b in range(B):
            m = n if count is None else int(count[b])
            m = m if 0 <= m <= n else 0
            assert bool((lp[b, m:] == 7).all()) and bool((ids[b, m:] == -7).all()), b
            if m == 0 or (B > 64 and b % 16 and b < B - 4):
                continue
            for i0 in range(0, m, 4096):
                i1 = min(m, i0 + 4096)
                x = z[b, i0:i1].double()
                want = x.log_softmax(-1)
                H = -(want.exp() * want).sum(-1)
                order = x.sort(dim=-1, descending=True, stable=True)[1][:, :5]
                assert bool(close(lp[b, i0:i1].double(), want.gather(-1, tokens[b, i0:i1, None].long())[:, 0], V).all()), (b, i0)
                assert bool(((ent[b, i0:i1].double() - H).abs() <= (2 * add + 16 * U) * (1 + H)).all()), (b, i0)
                assert torch.equal(ids[b, i0:i1].long(), order), (b, i0)
                assert bool(close(tl[b, i0:i1].double(), want.gather(-1, order), V).all()), (b, i0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tau", [1e-5, 3e-7, 1e-7, 1e-8, 1e-9, 1e-20, 1e-30, 1e-38, 1e20, 1e40, 1e60, 1e300])
def test_temperatures(tau, dtype):
    """Logits that the temperature takes past what fp32 tells apart, or past its range, or to
    nothing: one token takes all, or the equal ones do, or all that are not masked."""
    rng = np.random.default_rng(3)
    V, top = 5000, 8
    z = rng.standard_normal((1, 8, V), dtype=np.float32) * 8
    z[0, 1] -= 100                                    # a negative maximum
    z[0, 2, [7, 2500, 4999]] = 50.0                   # a shared one
    z[0, 3, rng.random(V) < 0.5] = -np.inf
    z[0, 4] *= 1e30
    z[0, 5] = -np.inf
    z[0, 6] = np.where(rng.random(V) < 0.5, torch.finfo(torch.bfloat16).min, -1e4 + z[0, 6])
    z[0, 7] = torch.finfo(torch.bfloat16).min
    Z = torch.from_numpy(z).to(torch.float32 if dtype == "f32" else torch.bfloat16).to(dev())
    zz = f64(Z)
    tokens = np.array([[int(np.argmax(zz[0, 0])), 11, 2500, 1, int(np.argmax(zz[0, 4])), 3, 4, 4999]], np.int32)
    tokens[0, 3] = int(np.nonzero(np.isinf(zz[0, 3]))[0][0])
    lp, ent, ids, tl = (t.cpu().numpy() for t in logprobs(Z, d_i32(tokens), tau=tau, top=top))
    add = (V / 64 + 96) * U
    near = lambda x, y: x == y or abs(x - y) <= add + 8 * U * (abs(y) + 1) or (y < -1e37 and x < -1e37)
    for i in range(8):
        want, H, order = ref.logprob_row(zz[0, i], tau)
        assert near(lp[0, i], want[tokens[0, i]]), (i, lp[0, i], want[tokens[0, i]])
        assert abs(ent[0, i] - H) <= (2 * add + 16 * U) * (1 + H), (i, ent[0, i], H)
        assert np.array_equal(ids[0, i], order[:top]), i
        assert all(near(x, want[o]) for x, o in zip(tl[0, i], order)), (i, tl[0, i], want[order[:top]])


# ------------------------------------------------------------------ capped scores
def capped_row(q, k, v, pos, scale, cap):
    """ref.attn_row without a window, its bound of a score's error for a cap that is taken with
    a relative error: 20 u (the fp32 factor of the cap 2 u; from 0.26 of the cap on the
    quotient's 16 u, below it the polynomial's few)."""
    w, o, lse, _, spread = ref.attn_row(q, k, v, pos, scale, cap, 0)
    x = k[:pos + 1] @ q * scale
    size = np.abs(k[:pos + 1]) @ np.abs(q) * scale
    return w, o, lse, (len(q) + 8) * U * size.max() + 20 * U * np.abs(cap * np.tanh(x / cap)).max(), spread


@pytest.mark.parametrize("G,D,dtype", [(4, 128, "bf16"), (12, 64, "e4m3"), (4, 64, "e4m3"), (12, 128, "bf16"), (3, 256, "bf16")])
@pytest.mark.parametrize("cap", [2.0 ** -20, 0.5, 8.0, 30.0, 1e4, 1e6, 1e8, 1e20, 2.0 ** 120, 2.0 ** 126])
def test_caps(cap, G, D, dtype):
    """Scores far below, around and far above the cap keep their digits, in the attention of few
    and of many rows and in the chosen heads' weights."""
    lens, n, heads = [150, 20], 5, 2
    c = Case(lens, n, heads * G, heads, D, 16, E4M3 if dtype == "e4m3" else torch.bfloat16, seed=G + D)
    out, L = c.attend(softcap=cap)
    row, chosen = [4, 0], list(range(heads * G))
    attn = torch.full((2, len(chosen), 160), 7.0, device=dev())
    pld.pld_cache_attn_rows(c.q, c.k, c.t, c.d_lens, d_i32(row), d_i32(chosen), L, attn, k_scale=c.ks, softcap=cap)
    out, lse, a = f64(out), f64(L), f64(attn)
    for b in range(2):
        for h in range(heads * G):
            k = ref.cache_rows(c.k, c.ks, c.table, b, h // G, lens[b] - 1 + n)
            v = ref.cache_rows(c.v, c.vs, c.table, b, h // G, lens[b] - 1 + n)
            for i in range(n):
                pos = lens[b] - 1 + i
                w, o, s, tol, spread = capped_row(f64(c.q[b, i, h]), k[:pos + 1], v[:pos + 1], pos, D ** -0.5, cap)
                assert abs(lse[b, i, h] - s) <= ref.lse_bound(tol, s, pos + 1), (b, i, h, lse[b, i, h], s)
                assert (np.abs(out[b, i, h] - o) <= ref.out_bound(o, spread, tol)).all(), (b, i, h)
                if i == row[b]:
                    w = w * np.exp(s - lse[b, i, h])
                    rel = np.expm1(2 * tol + 16 * U * (1 + abs(s) + np.abs(np.log(np.maximum(w, 1e-38)))))
                    assert (np.abs(a[b, h, :pos + 1] - w) <= rel * w + 2.0 ** -126).all(), (b, h)
                    assert (a[b, h, pos + 1:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("cap", [1.0, 10.0, 30.0])
@pytest.mark.parametrize("G", [1, 4, 12])
def test_capped_scores_go_by_their_own_keys(G, cap, dtype):
    """Large and infinite scores of keys that a row does not see leave its bits as they are,
    whichever form of the cap they take."""
    lens, n = [37, 130], 5
    c = Case(lens, n, 2 * G, 2, 64, 16, E4M3 if dtype == "e4m3" else torch.bfloat16, seed=G)
    c.q *= 4
    clean, L = c.attend(softcap=cap)
    used = np.zeros((c.k.shape[0], 16), bool)
    for b, T in enumerate(lens):
        for j in range(T + n - 1):
            used[c.table[b, j // 16], j % 16] = True
    hole = torch.from_numpy(~used).to(dev())
    for poison in (0.01, 30.0, 1e30, math.inf):
        if dtype == "bf16":
            c.k[hole] = poison
        else:
            c.ks.transpose(1, 2)[hole] = poison
        out, lse = c.attend(softcap=cap)
        assert np.array_equal(bits(out), bits(clean)) and np.array_equal(bits(lse), bits(L)), poison


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("cap", [0.0, 1000.0])
def test_weights_of_exact_products(cap, D):
    """Whole numbers, whose products are exact in fp32: what is left of a weight's error is that of
    the score's last roundings, of its distance d from the log sum (2.3 u of it: the difference and
    the product with log2(e), a constant off by 0.22 u) and of 2^x (2 u), and does not go with the
    score's size.  A capped score has its own 20 u."""
    c = Case([400, 77], 2, 8, 2, D, 16, seed=D)
    scale = float(np.float32(D ** -0.5))
    c.q = c.q.float().round().mul(2).to(torch.bfloat16)
    c.k = c.k.float().round().to(torch.bfloat16)
    row, lens = [1, 0], c.lens
    L, want = torch.zeros(2, 2, 8, device=dev()), {}
    for b in range(2):
        for h in range(8):
            x = ref.cache_rows(c.k, None, c.table, b, h // 4, lens[b] + row[b]) @ f64(c.q[b, row[b], h]) * scale
            x = cap * np.tanh(x / cap) if cap else x
            L[b, row[b], h] = float(np.logaddexp.reduce(x))
            want[b, h] = x - float(L[b, row[b], h]), np.abs(x)
    attn = torch.full((2, 8, 410), 7.0, device=dev())
    pld.pld_cache_attn_rows(c.q, c.k, c.t, c.d_lens, d_i32(row), d_i32(list(range(8))), L, attn, scale=scale, softcap=cap)
    a = f64(attn)
    for (b, h), (d, x) in want.items():
        rel = (2.5 * np.abs(d) + 4 + (21 * x if cap else 0)) * U
        assert x.max() > 4
        assert (np.abs(a[b, h, :len(d)] / np.exp(d) - 1) <= rel).all(), (b, h, (np.abs(a[b, h, :len(d)] / np.exp(d) - 1) / rel).max())


# ------------------------------------------------------------------ scales
@pytest.mark.parametrize("G", [1, 4, 12])            # 5, 20 and 60 rows a key head
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("which,poison", [("k", math.nan), ("v", math.nan), ("v", math.inf)])
def test_seen_scales_that_are_not_finite(which, poison, D, G):
    """A key's or value's scale that is NaN, or a value's that is infinite, at an early key that
    every row sees, reaches the output of every row of that key head, whatever their number, and
    no other's.  (An infinite scale of a key makes scores of either infinity, of which the
    negative one weighs nothing by its definition.)"""
    c = Case([400, 130], 5, 2 * G, 2, D, 16, E4M3, seed=D + G)
    clean, L = c.attend()
    scale = c.ks if which == "k" else c.vs
    scale[int(c.table[0, 2]), 1, 5] = poison
    out, _ = c.attend()
    assert np.array_equal(bits(out[1]), bits(clean[1])) and np.array_equal(bits(out[0, :, :G]), bits(clean[0, :, :G]))
    assert not torch.isfinite(out[0, :, G:].float()).any(-1).any()


# ------------------------------------------------------------------ large values
@pytest.mark.parametrize("G", [1, 4, 12])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_large_values(dtype, G):
    """Values of up to 2^89 and keys in the thousands: products are summed before the division by
    the weights' sum, and do not overflow."""
    c = Case([3000, 40], 5, 2 * G, 2, 128, 64, E4M3 if dtype == "e4m3" else torch.bfloat16, seed=G)
    if dtype == "bf16":
        c.v = (c.v.float().sign() * 2.0 ** 89).to(torch.bfloat16)
        c.v[:, :, 1] = 2.0 ** 89
    else:
        c.vs *= 2.0 ** 89 / (448 * 0.03)
    out, L = c.attend()
    c.check_attend(out, L, rows={(0, 0), (0, 4), (1, 0), (1, 3)})
    assert torch.isfinite(out.float()).all()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("size", [2.0 ** -60, 2.0 ** 59])
def test_norms_of_large_and_small_elements(size, D):
    """Norms of elements of one size, whose squares are near the ends of fp32: the signs times the
    weights, each rounded once (and the weights' products four times in fp32)."""
    c = Case([20], 3, 4, 2, D, 16, seed=D)
    sign = lambda *shape: (normal(c.rng, *shape).float() >= 0).float() * 2 - 1
    q, k, v = sign(1, 3, 4, D), sign(1, 3, 2, D), normal(c.rng, 1, 3, 2, D)
    w = normal(c.rng, D)
    out = torch.zeros_like(c.q)
    pld.pld_cache_write((q * size).to(torch.bfloat16), (k * size).to(torch.bfloat16), v, c.k, c.v, c.t, c.d_lens, out,
                        q_norm=w, k_norm=w, eps=0.0)
    stored = torch.stack([c.k[int(c.table[0, p // 16]), p % 16] for p in (19, 20, 21)])[None]
    for got, s in ((out, q), (stored, k)):
        want = f64(s) * f64(w)
        assert (np.abs(f64(got) - want) <= (2.0 ** -8 + 4 * U) * np.abs(want)).all()


# ------------------------------------------------------------------ wide strides
@pytest.mark.parametrize("D,G", [(128, 4), (64, 12)])      # 20 and 60 rows a key head
def test_slots_far_apart(D, G):
    """A page whose slots are so far apart that it spans more than 2^32 times 16 bytes (a cache
    that lies slot by slot): what the write puts there, the attention and the chosen heads'
    weights read.  The same rows in a cache of ordinary strides give the same bits."""
    page, heads, T, slot = 4096, 2, 4090, 9 << 20
    size = (page - 1) * slot + 2 * heads * D
    assert (page - 16) * (slot * 2 // 16) > 2 ** 32
    if torch.cuda.mem_get_info()[0] < 2 * size + (4 << 30):
        pytest.skip("too little memory is free")
    near = Case([T], 5, heads * G, heads, D, page, seed=D)
    flat = torch.empty(size, dtype=torch.bfloat16, device=dev())        # values beside keys
    far = [flat.as_strided((1, page, heads, D), (page * slot, slot, D, 1), at) for at in (0, heads * D)]
    for x, old in zip(far, (near.k, near.v)):
        x[0].copy_(old[int(near.table[0, 0])])
    table = torch.zeros((1, 1), dtype=torch.int32, device=dev())
    k, v = normal(near.rng, 1, 5, heads, D), normal(near.rng, 1, 5, heads, D)
    got = []
    for kc, vc, t in ((near.k, near.v, near.t), (far[0], far[1], table)):
        q, out, L = torch.empty_like(near.q), torch.zeros_like(near.q), torch.zeros((1, 5, heads * G), device=dev())
        attn = torch.zeros((1, 3, page), device=dev())
        ws = torch.zeros(pld.pld_cache_attn_workspace_bytes(1, 5, heads * G, heads, D), dtype=torch.uint8, device=dev())
        pld.pld_cache_write(near.q, k, v, kc, vc, t, near.d_lens, q)
        pld.pld_cache_attn(q, kc, vc, t, near.d_lens, out, ws, lse=L)
        pld.pld_cache_attn_rows(q, kc, t, near.d_lens, d_i32([4]), d_i32([0, G, G + 1]), L, attn)
        got.append([bits(x) for x in (q, out, L, attn)])
    del flat, far, kc, vc, x
    torch.cuda.empty_cache()
    for a, b in zip(*got):
        assert np.array_equal(a, b)
    near.check_attend(out, L)


# ------------------------------------------------------------------ another stream
@pytest.mark.parametrize("handle", [False, True])
def test_a_workspace_comes_from_the_stream_that_uses_it(handle, monkeypatch):
    """attend() on another stream than the current one allocates its workspace under that
    stream, not from memory that the current stream's earlier work may still be using."""
    cache = PagedCache(1, 5000, 2, 64, page_size=16)
    rng = np.random.default_rng(4)
    for x in (cache.k, cache.v):
        x.copy_(normal(rng, *x.shape))
    q, lens = normal(rng, 1, 3, 8, 64), d_i32([4900])
    want, out = torch.zeros_like(q), torch.zeros_like(q)
    cache.attend(q, lens, want)
    fresh = PagedCache(1, 5000, 2, 64, page_size=16)
    fresh.k, fresh.v, fresh.table = cache.k, cache.v, cache.table
    side, under, empty = torch.cuda.Stream(), [], torch.empty
    torch.cuda.synchronize()
    monkeypatch.setattr(torch, "empty", lambda *a, **k: (under.append(torch.cuda.current_stream().cuda_stream), empty(*a, **k))[1])
    fresh.attend(q, lens, out, stream=side.cuda_stream if handle else side)
    monkeypatch.undo()
    assert under == [side.cuda_stream] and torch.cuda.current_stream() != side
    side.synchronize()
    assert np.array_equal(bits(out), bits(want))


def test_a_workspace_for_the_default_stream(monkeypatch):
    """The default stream's handle is 0."""
    cache, under, empty = PagedCache(1, 100, 2, 64, page_size=16), [], torch.empty
    q, lens = torch.zeros((1, 3, 8, 64), dtype=torch.bfloat16, device=dev()), d_i32([50])
    torch.cuda.synchronize()
    monkeypatch.setattr(torch, "empty", lambda *a, **k: (under.append(torch.cuda.current_stream().cuda_stream), empty(*a, **k))[1])
    with torch.cuda.stream(torch.cuda.Stream()):
        cache.attend(q, lens, torch.zeros_like(q), stream=0)
    monkeypatch.undo()
    assert under == [0]
    torch.cuda.synchronize()
