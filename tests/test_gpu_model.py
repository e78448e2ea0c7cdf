"""The model-side calls of a verification pass against plain 64-bit references (model_ref.py).

The paged cache's write, the attention over it, the attention rows of chosen heads and the
tokens' log probabilities, at the sizes, masks, strides and faults where they can go wrong;
then a generation loop of them all.  Bounds come from the arithmetic: see model_ref.py.
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
from paper_2412_01447_amd.step import DraftStep, decode_loop

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn
NAN = math.nan


def normal(rng, *shape, gain=1.0):
    x = rng.standard_normal(shape, dtype=np.float32) * gain
    return torch.from_numpy(x).to(torch.bfloat16).to(dev())


def bits(t):
    t = t.contiguous()
    return t.view(torch.uint8).cpu().numpy() if t.dtype == E4M3 else \
        t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).cpu().numpy()


class Case:
    """A cache filled with values, its pages in a random order, and rows of queries."""

    def __init__(self, lens, n, Hq, heads, D, page=16, dtype=torch.bfloat16, draft_len=None,
                 layout="slots", extra=2, seed=0, gain=2.0):
        self.rng = rng = np.random.default_rng(seed)
        B = len(lens)
        self.lens, self.n, self.Hq, self.heads, self.D, self.page = lens, n, Hq, heads, D, page
        self.dl = draft_len
        per = max(1, -(-(max(lens) + n) // page))
        P = B * per + extra
        self.table = rng.permutation(P)[:B * per].reshape(B, per).astype(np.int32)
        k, v = normal(rng, P, page, heads, D), normal(rng, P, page, heads, D)
        self.ks = self.vs = None
        if dtype == E4M3:
            self.ks = torch.from_numpy(rng.uniform(0.01, 0.03, (P, heads, page)).astype(np.float32)).to(dev())
            self.vs = torch.from_numpy(rng.uniform(0.01, 0.03, (P, heads, page)).astype(np.float32)).to(dev())
            k, v = (k.float() * 64).to(E4M3), (v.float() * 64).to(E4M3)
        if layout == "heads":            # [page][head][slot][t]
            k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
        elif layout == "pairs":          # keys and values side by side, page by page
            both = torch.stack([k, v], 1)
            k, v = both[:, 0], both[:, 1]
        self.k, self.v = k, v
        self.q = normal(rng, B, n, Hq, D, gain=gain)
        self.t = d_i32(self.table)
        self.d_lens = d_i32(lens)
        self.d_dl = None if draft_len is None else d_i32(draft_len)

    def attend(self, softcap=0.0, window=0, scale=None, q=None, lse=True, stream=None):
        B = len(self.lens)
        q = self.q if q is None else q
        out = torch.full((B, self.n, self.Hq, self.D), 7.0, dtype=torch.bfloat16, device=dev())
        L = torch.full((B, self.n, self.Hq), 7.0, device=dev()) if lse else None
        need = pld.pld_cache_attn_workspace_bytes(B, self.n, self.Hq, self.heads, self.D)
        ws = torch.full((need,), 0x7f, dtype=torch.uint8, device=dev())
        pld.pld_cache_attn(q, self.k, self.v, self.t, self.d_lens, out, ws, draft_len=self.d_dl,
                           k_scale=self.ks, v_scale=self.vs, lse=L, scale=scale, softcap=softcap,
                           window=window, stream=stream)
        return out, L

    def check_attend(self, out, L, softcap=0.0, window=0, scale=None, rows=None):
        """rows: (b, i) pairs to check; the others only for being written where they exist."""
        out, L = f64(out), None if L is None else L.cpu().numpy()
        scale = self.D ** -0.5 if scale is None else scale
        for b in range(len(self.lens)):
            cnt, p0 = ref.rows_of(self.lens, self.dl, self.n, b)
            assert np.all(out[b, cnt:] == 7.0) and (L is None or np.all(L[b, cnt:] == 7.0)), b
            if cnt == 0:
                continue
            todo = [i for i in range(cnt) if rows is None or (b, i) in rows]
            for kv in range(self.heads) if todo else ():
                k = ref.cache_rows(self.k, self.ks, self.table, b, kv, p0 + cnt)
                v = ref.cache_rows(self.v, self.vs, self.table, b, kv, p0 + cnt)
                G = self.Hq // self.heads
                for i in todo:
                    for h in range(kv * G, kv * G + G):
                        _, o, lse, tol, spread = ref.attn_row(
                            f64(self.q[b, i, h]), k[:p0 + i + 1], v[:p0 + i + 1], p0 + i, scale,
                            softcap, window)
                        if math.isnan(lse):
                            assert np.isnan(out[b, i, h]).all(), (b, i, h)
                            assert L is None or np.isnan(L[b, i, h]), (b, i, h)
                            continue
                        off = np.abs(out[b, i, h] - o) - ref.out_bound(o, spread, tol)
                        assert off.max() <= 0, (b, i, h, off.max())
                        if L is not None:
                            assert abs(L[b, i, h] - lse) <= ref.lse_bound(tol, lse, p0 + i + 1), \
                                (b, i, h, L[b, i, h], lse)


# ------------------------------------------------------------------ attention
ATTEND = [
    # lens, n, Hq, heads, D, page, dtype, layout, softcap, window, draft_len
    ([1], 1, 1, 1, 64, 16, "bf16", "slots", 0, 0, None),
    ([1, 2, 3], 2, 4, 4, 128, 16, "bf16", "slots", 0, 0, None),
    ([15, 16, 17, 31], 3, 8, 2, 64, 16, "bf16", "heads", 0, 0, [2, 0, 1, 2]),
    ([33, 64, 127, 128, 129], 5, 8, 1, 128, 32, "bf16", "pairs", 0, 0, [4, 3, 2, 1, 0]),
    ([500, 1, 77], 17, 12, 4, 128, 64, "bf16", "slots", 0, 0, None),
    ([700, 300], 11, 40, 8, 64, 16, "bf16", "slots", 0, 0, [10, 4]),
    ([260, 90], 4, 6, 2, 256, 32, "bf16", "slots", 0, 0, None),
    ([1000, 257], 7, 16, 2, 128, 128, "bf16", "slots", 30.0, 0, None),
    ([1000, 5, 63], 9, 4, 2, 64, 16, "bf16", "slots", 0, 1, None),
    ([1000, 65, 200], 9, 8, 2, 128, 16, "bf16", "slots", 0, 37, [8, 8, 3]),
    ([400, 399], 6, 4, 1, 256, 16, "bf16", "heads", 50.0, 200, None),
    ([300, 17], 3, 8, 2, 128, 16, "e4m3", "slots", 0, 0, None),
    ([513, 100], 17, 16, 2, 64, 32, "e4m3", "heads", 0, 64, [16, 5]),
    ([200, 130], 2, 10, 2, 256, 64, "e4m3", "pairs", 20.0, 0, None),
    ([90, 4], 71, 8, 2, 128, 16, "bf16", "slots", 0, 0, [70, 64]),
    ([2049], 33, 16, 1, 128, 4096, "bf16", "slots", 0, 0, None),
    ([300, 64, 1], 9, 8, 1, 128, 16, "bf16", "heads", 0, 0, [8, 3, 8]),     # 5 tiles of 16 rows
    ([300, 90], 17, 16, 2, 128, 16, "e4m3", "pairs", 0, 70, [16, 4]),       # 9 and 3
    ([140], 22, 8, 1, 64, 16, "e4m3", "slots", 25.0, 0, None),              # 11
    ([140, 20], 23, 8, 1, 64, 32, "bf16", "slots", 0, 0, [22, 1]),          # 12: two groups
    ([150, 33], 17, 16, 2, 256, 16, "bf16", "slots", 0, 40, None),          # 9, of heads of 256
    ([150, 33], 8, 8, 1, 256, 16, "e4m3", "slots", 0, 0, [7, 5]),
    ([600], 200, 4, 2, 128, 64, "bf16", "slots", 0, 100, None),             # a prompt's chunk
]


@pytest.mark.parametrize("lens,n,Hq,heads,D,page,dtype,layout,softcap,window,dl", ATTEND)
def test_attend(lens, n, Hq, heads, D, page, dtype, layout, softcap, window, dl):
    c = Case(lens, n, Hq, heads, D, page, E4M3 if dtype == "e4m3" else torch.bfloat16, dl, layout,
             seed=len(lens) * n + D)
    say("attend", lens, n, Hq, heads, D, page, dtype, layout, softcap, window)
    out, L = c.attend(softcap, window)
    torch.cuda.synchronize()
    c.check_attend(out, L, softcap, window)
    again, L2 = c.attend(softcap, window)
    assert np.array_equal(bits(out), bits(again)) and np.array_equal(bits(L), bits(L2))
    bare, _ = c.attend(softcap, window, lse=False)
    assert np.array_equal(bits(out), bits(bare))


@pytest.mark.parametrize("D,heads,G,dtype", [(128, 8, 4, "bf16"), (64, 2, 8, "e4m3"),
                                             (128, 1, 16, "e4m3"), (256, 1, 1, "bf16"),
                                             (128, 2, 36, "bf16"), (128, 1, 44, "e4m3"),
                                             (64, 1, 24, "bf16"), (256, 1, 24, "e4m3")])
def test_attend_long(D, heads, G, dtype):
    """Tens of thousands of keys split over many blocks beside short sequences; a sample of
    the rows is checked, all of them for being written."""
    lens = [40001, 3, 8192, 20000]
    c = Case(lens, 4, heads * G, heads, D, 64, E4M3 if dtype == "e4m3" else torch.bfloat16,
             [3, 3, 0, 2], seed=D)
    out, L = c.attend()
    c.check_attend(out, L, rows={(0, 0), (0, 3), (1, 1), (2, 0), (3, 2)})
    assert not torch.isnan(out).any()


def test_attend_large_batch():
    """More sequences than blocks fit on the GPU at once, lengths of every size."""
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 300, 700).astype(np.int32)
    dl = rng.integers(-1, 4, 700).astype(np.int32)      # -1 and 3 (= n) name no rows
    c = Case(lens, 3, 4, 2, 64, 32, draft_len=dl, seed=6)
    out, L = c.attend()
    c.check_attend(out, L, rows={(int(b), int(i)) for b, i in zip(rng.integers(0, 700, 90), rng.integers(0, 3, 90))})


def test_largest_batch_of_single_tokens():
    """65535 sequences of one token: the only key's value is the output, bit for bit, and its
    score the log sum; then the same keys' weights, all 1."""
    B, D = 65535, 64
    rng = np.random.default_rng(4)
    q, k, v = (normal(rng, B, 1, 1, D) for _ in range(3))
    cache = PagedCache(B, 16, 1, D, page_size=16)
    lens, q_out = torch.ones(B, dtype=torch.int32, device=dev()), torch.zeros_like(q)
    cache.write(q, k, v, lens, q_out)
    assert np.array_equal(bits(q_out), bits(q))
    assert np.array_equal(bits(cache.k[:, 0]), bits(k[:, 0])) and np.array_equal(bits(cache.v[:, 0]), bits(v[:, 0]))
    assert not cache.k[:, 1:].any() and not cache.v[:, 1:].any()
    out, L = torch.zeros_like(q), torch.zeros((B, 1, 1), device=dev())
    cache.attend(q, lens, out, lse=L)
    assert np.array_equal(bits(out), bits(v))
    x = (f64(q) * f64(k)).sum(-1) / 8
    tol = (D + 8) * U * (np.abs(f64(q)) * np.abs(f64(k))).sum(-1) / 8
    assert (np.abs(f64(L) - x) <= ref.lse_bound(tol, x, 1)).all()
    attn = torch.full((B, 1, 3), 7.0, device=dev())
    cache.weights(q, lens, torch.zeros_like(lens), d_i32([0]), L, attn)
    a = f64(attn)
    assert (np.abs(a[:, :, 0] - 1) <= np.expm1(2 * tol + 16 * U * (1 + np.abs(x)))[:, 0]).all() and (a[:, :, 1:] == 7).all()


@pytest.mark.parametrize("G,D,window,dtype", [(8, 64, 0, "bf16"), (1, 128, 300, "bf16"), (12, 64, 100, "e4m3")])
def test_prompt_chunk(G, D, window, dtype):
    """Thousands of rows a sequence, in many groups; a sample of them is checked."""
    n = 3000
    c = Case([1, 500], n, G, 1, D, 64, E4M3 if dtype == "e4m3" else torch.bfloat16, [n - 1, 1700], seed=G)
    out, L = c.attend(window=window)
    rows = {(0, 0), (0, 1), (0, 17), (0, 1499), (0, 2998), (0, 2999), (1, 0), (1, 333), (1, 1700)}
    c.check_attend(out, L, window=window, rows=rows)
    assert not torch.isnan(out.float()).any()


@pytest.mark.parametrize("Hq,heads", [(4096, 1), (1024, 1024), (4096, 512)])
def test_most_heads(Hq, heads):
    """The most query heads a key head, and the most key heads, through all of the cache's calls."""
    lens, n, D = [19, 40], 2, 64
    c = Case(lens, n, Hq, heads, D, 16, draft_len=[1, 0], seed=Hq + heads)
    k, v = normal(c.rng, 2, n, heads, D), normal(c.rng, 2, n, heads, D)
    q = torch.zeros_like(c.q)
    pld.pld_cache_write(c.q, k, v, c.k, c.v, c.t, c.d_lens, q, draft_len=c.d_dl)
    for b, cnt in ((0, 2), (1, 1)):
        assert np.array_equal(bits(q[b, :cnt]), bits(c.q[b, :cnt])) and not q[b, cnt:].any()
        for i in range(cnt):
            p = lens[b] - 1 + i
            at = int(c.table[b, p // 16]), p % 16
            assert np.array_equal(bits(c.k[at]), bits(k[b, i])) and np.array_equal(bits(c.v[at]), bits(v[b, i]))
    out, L = c.attend()
    c.check_attend(out, L, rows={(0, 1), (1, 0)})
    chosen = [Hq - 1, 0, Hq // 2, Hq - 1, Hq // 3]
    attn = torch.full((2, 5, 41), 7.0, device=dev())
    pld.pld_cache_attn_rows(c.q, c.k, c.t, c.d_lens, d_i32([1, 0]), d_i32(chosen), L, attn)
    a, lse = f64(attn), f64(L)
    for b, i in ((0, 1), (1, 0)):
        p = lens[b] - 1 + i
        assert (a[b, :, p + 1:] == 7).all()
        for r, h in enumerate(chosen):
            kk = ref.cache_rows(c.k, None, c.table, b, h // (Hq // heads), p + 1)
            x = kk @ f64(c.q[b, i, h]) / 8
            tol = (D + 8) * U * (np.abs(kk) @ np.abs(f64(c.q[b, i, h]))).max() / 8
            w = np.exp(x - lse[b, i, h])
            bound = np.expm1(2 * tol + 16 * U * (1 + abs(lse[b, i, h]) + np.abs(x - lse[b, i, h]))) * w + 2.0 ** -126
            assert (np.abs(a[b, r, :p + 1] - w) <= bound).all(), (b, r)


def test_shared_pages():
    """Sequences that share their first pages, one of them with a page twice, read the same rows."""
    c = Case([64, 64, 50], 1, 8, 2, 64, 16, seed=9)
    c.table[1, :3] = c.table[0, :3]
    c.table[2, :3] = c.table[0, 0]
    c.t = d_i32(c.table)
    out, L = c.attend()
    c.check_attend(out, L)


def test_nothing_to_do():
    """No sequence has a row: nothing is written, and the workspace serves the next call."""
    c = Case([5, 0, 9], 2, 8, 2, 64, 16, draft_len=[-1, 1, 2], seed=9)
    out, L = c.attend()
    assert (out == 7).all() and (L == 7).all()
    attn = torch.full((3, 1, 12), 7.0, device=dev())
    pld.pld_cache_attn_rows(c.q, c.k, c.t, c.d_lens, d_i32([-1, 0, 2]), d_i32([0]), L, attn)
    assert (attn == 7).all()
    z, lp = torch.zeros(3, 2, 100, device=dev()), torch.full((3, 2), 7.0, device=dev())
    ids, tl = torch.full((3, 2, 4), -7, dtype=torch.int32, device=dev()), torch.full((3, 2, 4), 7.0, device=dev())
    ws = torch.zeros(pld.pld_token_logprobs_workspace_bytes(3, 2, 100, pld.PLD_F32, 4), dtype=torch.uint8, device=dev())
    pld.pld_token_logprobs(z, d_i32(np.zeros((3, 2))), lp, ws, count=d_i32([0, -1, 3]), top_ids=ids, top_logprobs=tl)
    assert (lp == 7).all() and (ids == -7).all() and (tl == 7).all()


def test_attend_spread_scores():
    """Scores thousands apart (one key takes all), equal keys, and a head of zeros."""
    c = Case([300, 40], 2, 8, 2, 128, 16, seed=3, gain=60.0)
    c.q[0, 1] = 0
    c.k[:, :, 1] = c.k[0, 0, 1]
    out, L = c.attend()
    c.check_attend(out, L)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("poison", [NAN, math.inf, -math.inf])
@pytest.mark.parametrize("G", [1, 4, 12])        # 5, 20 and 60 rows a key head
def test_attend_masked_places(dtype, window, poison, G):
    """What stands in slots that a row does not see -- past its position (other rows' slots
    among them), before its window, on unused pages -- does not reach it."""
    lens, n = [37, 1, 130], 5
    c = Case(lens, n, 2 * G, 2, 64, 16, E4M3 if dtype == "e4m3" else torch.bfloat16, [4, 2, 4], seed=11)
    P = c.k.shape[0]
    used = np.zeros((P, 16), bool)
    for b, T in enumerate(lens):
        cnt, p0 = ref.rows_of(c.lens, c.dl, n, b)
        lo = max(0, p0 + 1 - window) if window else 0
        for j in range(lo, p0 + cnt):
            used[c.table[b, j // 16], j % 16] = True
    hole = torch.from_numpy(~used).to(dev())
    bad = torch.tensor(poison, device=dev()).to(torch.bfloat16)
    if dtype == "bf16":
        c.k[hole], c.v[hole] = bad, bad
    else:
        # e4m3 has no infinity: its NaN, and scales of the poison
        for x in (c.k, c.v):
            x.view(torch.uint8)[hole] = 0x7f
        c.ks.transpose(1, 2)[hole], c.vs.transpose(1, 2)[hole] = poison, poison
    out, L = c.attend(window=window)
    c.check_attend(out, L, window=window)
    # a later row's own value: the rows before it do not see it, it and the rows after do
    b, i = 2, 2
    slot = lens[b] - 1 + i
    at = int(c.table[b, slot // 16]), slot % 16
    if dtype == "bf16":
        c.v[at] = bad
    else:
        c.vs[at[0], :, at[1]] = poison
    got, _ = c.attend(window=window)
    assert np.array_equal(bits(got[0]), bits(out[0])) and np.array_equal(bits(got[1]), bits(out[1]))
    c.check_attend(got[:, :], L, window=window, rows={(b, 0), (b, 1)})
    assert not torch.isfinite(got[b, 2:].float()).any()
    # and before the window of the later rows
    if window:
        first = lens[0] - window            # row 0 sees it, row 1 does not
        at = int(c.table[0, first // 16]), first % 16
        if dtype == "bf16":
            c.v[at] = bad
        else:
            c.vs[at[0], :, at[1]] = poison
        got, _ = c.attend(window=window)
        assert not torch.isfinite(got[0, 0].float()).any()
        for i in range(1, 5):
            assert np.array_equal(bits(got[0, i]), bits(out[0, i])), i


@pytest.mark.parametrize("G", [4, 12])
def test_attend_bad_pages_and_ends(G):
    """A bad page gives NaN to the rows that see it and to no others; rows past the table are
    NaN; sequences without rows are left alone."""
    c = Case([100, 100, 100, 0, 50, 31], 4, 2 * G, 2, 64, 16, draft_len=[3, 3, 3, 3, 4, -1], seed=2)
    c.table[0, 3] = -1
    c.table[1, 0] = c.k.shape[0]
    c.t = d_i32(c.table)
    out, L = c.attend()
    c.check_attend(out, L)
    assert torch.isnan(out[:2].float()).all() and torch.isnan(L[:2]).all()
    assert not torch.isnan(out[2:].float()).any()
    # only through the window
    out, L = c.attend(window=30)
    c.check_attend(out, L, window=30)
    assert not torch.isnan(out.float()).any()
    # a table that ends inside the rows, or before them
    c = Case([30, 30, 30, 30], 4, 2 * G, 2, 64, 16, seed=2)
    c.lens = [30, 47, 200, 2 ** 31 - 1]
    c.d_lens = d_i32(c.lens)
    out, L = c.attend()
    cap = c.table.shape[1] * 16
    for b in range(4):
        for i in range(4):
            gone = c.lens[b] - 1 + i >= cap
            assert bool(torch.isnan(out[b, i].float()).all()) == gone, (b, i)
            assert bool(torch.isnan(L[b, i]).all()) == gone, (b, i)
            assert bool(torch.isnan(out[b, i].float()).any()) == gone, (b, i)


def test_attend_strides_and_offsets():
    """Queries inside a wider projection, outputs inside a wider buffer, rows before sequences,
    a table with room to spare, and a cache past 2^31 elements."""
    c = Case([70, 200], 3, 8, 2, 128, 16, seed=8)
    wide = normal(c.rng, 2, 3, 12 * 128)
    c.q = wide[:, :, 2 * 128:10 * 128].unflatten(-1, (8, 128))
    out, L = c.attend()
    c.check_attend(out, L)
    turned = c.q.transpose(0, 1).contiguous().transpose(0, 1)
    same, _ = c.attend(q=turned)
    assert np.array_equal(bits(out), bits(same))
    big = torch.full((2, 3, 10, 128), 7.0, dtype=torch.bfloat16, device=dev())
    ws = torch.zeros(pld.pld_cache_attn_workspace_bytes(2, 3, 8, 2, 128), dtype=torch.uint8, device=dev())
    t = torch.full((2, c.table.shape[1] + 5), -1, dtype=torch.int32, device=dev())
    t[:, :c.table.shape[1]] = c.t
    pld.pld_cache_attn(c.q, c.k, c.v, t[:, :c.table.shape[1]], c.d_lens, big[:, :, 1:9], ws)
    assert np.array_equal(bits(out), bits(big[:, :, 1:9]))
    assert (big[:, :, 0] == 7).all() and (big[:, :, 9] == 7).all()
    # 2^31 elements and more between pages: 9 GB of keys and values, the last pages used
    P, page = 70000, 64
    k = torch.zeros((P, page, 4, 128), dtype=torch.bfloat16, device=dev())
    v = torch.zeros_like(k)
    far = np.arange(P - c.table.size, P, dtype=np.int32).reshape(c.table.shape)
    w = Case([70, 200], 3, 8, 4, 128, 64, seed=9)
    far = np.arange(P - w.table.size, P, dtype=np.int32)[::-1].reshape(w.table.shape).copy()
    k[torch.from_numpy(far).long().to(dev())] = w.k[w.t.long()]
    v[torch.from_numpy(far).long().to(dev())] = w.v[w.t.long()]
    a, la = w.attend()
    w.k, w.v, w.table, w.t = k, v, far, d_i32(far)
    b, lb = w.attend()
    assert np.array_equal(bits(a), bits(b)) and np.array_equal(bits(la), bits(lb))


# ------------------------------------------------------------------ write
WRITE = [
    # lens, n, Hq, heads, D, page, dtype, layout, rot, pairs, norm, draft_len
    ([1], 1, 1, 1, 64, 16, "bf16", "slots", 64, "halves", True, None),
    ([5, 0, 31], 4, 8, 2, 128, 16, "bf16", "slots", 128, "halves", True, [3, 3, 1]),
    ([16, 17], 3, 5, 5, 128, 16, "bf16", "heads", 64, "neighbours", False, None),
    ([100, 1], 2, 12, 4, 256, 32, "bf16", "pairs", 256, "halves", False, None),
    ([9], 40, 6, 2, 64, 16, "bf16", "slots", 8, "halves", True, None),
    ([9, 60], 7, 6, 2, 64, 16, "bf16", "slots", 24, "neighbours", True, None),
    ([64, 3, 4], 17, 16, 2, 128, 64, "e4m3", "slots", 128, "halves", True, [16, -1, 17]),
    ([30, 3], 5, 4, 1, 256, 16, "e4m3", "heads", 128, "neighbours", False, None),
    ([30, 3], 5, 4, 4, 64, 16, "e4m3", "pairs", 0, "halves", False, [2, 4]),
    ([2], 300, 40, 8, 128, 128, "bf16", "slots", 0, "halves", True, None),
]


@pytest.mark.parametrize("lens,n,Hq,heads,D,page,dtype,layout,rot,pairs,norm,dl", WRITE)
@pytest.mark.parametrize("fused", [False, True])
def test_write(lens, n, Hq, heads, D, page, dtype, layout, rot, pairs, norm, dl, fused):
    c = Case(lens, n, Hq, heads, D, page, E4M3 if dtype == "e4m3" else torch.bfloat16, dl, layout,
             seed=n + D)
    B, rng = len(lens), c.rng
    say("write", lens, n, Hq, heads, D, page, dtype, layout, rot, pairs, norm, fused)
    k, v = normal(rng, B, n, heads, D), normal(rng, B, n, heads, D)
    q = c.q
    if fused:
        x = torch.cat([t.flatten(2) for t in (q, k, v)], -1)
        q, k, v = (t.unflatten(-1, (-1, D)) for t in x.split([Hq * D, heads * D, heads * D], -1))
    qw = kw = rope = None
    if norm:
        qw, kw = normal(rng, D), normal(rng, D)
    if rot:
        rope = torch.from_numpy(rng.uniform(-1, 1, (max(lens) + n, rot)).astype(np.float32)).to(dev())
    before = [None if t is None else bits(t).copy() for t in (c.k, c.v, c.ks, c.vs)]
    out = torch.full((B, n, Hq, D), 7.0, dtype=torch.bfloat16, device=dev())
    eps = 1e-5
    pld.pld_cache_write(q, k, v, c.k, c.v, c.t, c.d_lens, out, draft_len=c.d_dl, k_scale=c.ks,
                        v_scale=c.vs, q_norm=qw, k_norm=kw, eps=eps, rope=rope,
                        rope_pairs=pld.PLD_ROPE_HALVES if pairs == "halves" else pld.PLD_ROPE_NEIGHBOURS)
    got = f64(out)
    R = None if rope is None else f64(rope)
    touched = np.zeros((c.k.shape[0], page), bool)
    for b in range(B):
        cnt, p0 = ref.rows_of(lens, dl, n, b)
        assert np.all(got[b, cnt:] == 7.0)
        for i in range(cnt):
            pos = p0 + i
            at = int(c.table[b, pos // page]), pos % page
            touched[at] = True
            for src, w, dst in ((q, qw, None), (k, kw, c.k), (v, None, c.v)):
                x = ref.normed(f64(src[b, i]), None if w is None else f64(w), eps)
                y = x if src is v else ref.turned(x, R, pos, pairs == "halves")
                # the norm's sum and quotients (D + 16 roundings), the turn's products
                fp32 = (D + 24) * U * (np.abs(x).max(-1, keepdims=True) * 2 + 1e-30)
                if dst is None or dtype == "bf16":
                    z = got[b, i] if dst is None else f64(dst[at])
                    off = np.abs(z - y) - (2.0 ** -8 * np.abs(y) + fp32)
                else:
                    sc = f64((c.ks if src is k else c.vs)[at[0], :, at[1]])[:, None]
                    want = np.abs(y).max(-1, keepdims=True) / 448
                    assert (np.abs(sc - want) <= fp32 / 448 + 4 * U * want).all(), (b, i)
                    # half a step of a normal number, of the smallest one below
                    off = np.abs(f64(dst[at]) * sc - y) - (2.0 ** -4 * np.abs(y) + 2.0 ** -10 * sc + 2 * fp32)
                assert off.max() <= 0, (b, i, off.max())
    for t, old in zip((c.k, c.v, c.ks, c.vs), before):
        if t is not None:
            rest = torch.from_numpy(~touched)
            new = bits(t)
            if t.dim() == 3:
                new, old = new.transpose(0, 2, 1), old.transpose(0, 2, 1)
            assert np.array_equal(new[rest.numpy()], old[rest.numpy()])


def test_write_in_place_bad_pages_and_ends():
    """q_out = q; rows on bad pages, past the table or past the angles are not stored and
    their queries are NaN."""
    c = Case([30, 30, 30], 4, 4, 2, 64, 16, seed=4)
    k, v = normal(c.rng, 3, 4, 2, 64), normal(c.rng, 3, 4, 2, 64)
    rope = torch.from_numpy(c.rng.uniform(-1, 1, (33, 64)).astype(np.float32)).to(dev())
    apart = torch.zeros_like(c.q)
    pld.pld_cache_write(c.q, k, v, c.k, c.v, c.t, c.d_lens, apart, rope=rope)
    q = c.q.clone()
    pld.pld_cache_write(q, k, v, c.k, c.v, c.t, c.d_lens, q, rope=rope)
    assert np.array_equal(bits(q), bits(apart))
    old = bits(c.k).copy()
    c.table[1, 1] = 10 ** 9
    c.table[2, 2] = -5
    lens = [31, 14, 2 ** 31 - 1]
    q = c.q.clone()
    pld.pld_cache_write(q, k * 2, v, c.k, c.v, d_i32(c.table), d_i32(lens), q, rope=rope)
    nan = torch.isnan(q.float()).all(-1).all(-1).cpu().numpy()
    assert nan.tolist() == [[False, False, False, True],          # positions 30..33, 33 angles
                            [False, False, False, True],          # positions 13..16, page 1 bad
                            [True, True, True, True]]
    touched = {(int(c.table[b, p // 16]), p % 16) for b, p in ((0, 30), (0, 31), (0, 32), (1, 13), (1, 14), (1, 15))}
    new = bits(c.k)
    for pg in range(new.shape[0]):
        for s in range(16):
            assert np.array_equal(new[pg, s], old[pg, s]) == ((pg, s) not in touched), (pg, s)


def test_write_e4m3_scales():
    """Rows of zeros, of one tiny value, of the type's largest, and of infinities."""
    D = 64
    c = Case([1], 5, 1, 1, D, 16, E4M3, seed=1)
    k = torch.zeros((1, 5, 1, D), dtype=torch.bfloat16, device=dev())
    k[0, 1, 0, 3] = 2.0 ** -130
    k[0, 2] = torch.finfo(torch.bfloat16).max
    k[0, 3, 0, 0], k[0, 3, 0, 1] = 448.0, 2.0 ** -9
    k[0, 4, 0, 5] = math.inf
    out = torch.empty_like(c.q)
    pld.pld_cache_write(c.q, k, k, c.k, c.v, c.t, c.d_lens, out, k_scale=c.ks, v_scale=c.vs)
    pg = int(c.table[0, 0])
    got, sc = f64(c.k[pg, :5, 0]), f64(c.ks[pg, 0, :5])
    assert np.array_equal(bits(c.k[pg, :5]), bits(c.v[pg, :5]))
    assert (got[0] == 0).all() and sc[0] == 2.0 ** -126
    assert sc[1] == 2.0 ** -126 and got[1, 3] * sc[1] == 2.0 ** -130
    assert (got[2] == 448).all() and abs(sc[2] * 448 / float(torch.finfo(torch.bfloat16).max) - 1) < 4 * U
    assert sc[3] == 1 and got[3, 0] == 448 and got[3, 1] == 2.0 ** -9
    with np.errstate(invalid="ignore"):
        assert np.isnan(got[4] * sc[4]).all()


# ------------------------------------------------------------------ rows
ROWS = [
    # lens, n, Hq, heads, D, page, dtype, softcap, window, rows, chosen, n_keys short of the rows
    ([1, 2], 1, 1, 1, 64, 16, "bf16", 0, 0, [0, 0], [0], 0),
    ([40, 300, 17], 5, 8, 2, 128, 16, "bf16", 0, 0, [4, 0, 2], [7, 0, 3, 3], 0),
    ([40, 1000, 64], 3, 40, 8, 64, 32, "bf16", 0, 0, [2, 1, 0], list(range(40)), 0),
    ([40, 300, 17], 5, 12, 4, 128, 16, "e4m3", 30.0, 0, [4, -1, 5], [11, 2], 0),
    ([90, 257], 4, 6, 1, 256, 64, "e4m3", 0, 50, [3, 0], [5, 1, 2, 0, 4], 0),
    ([500, 100], 2, 64, 1, 128, 16, "bf16", 0, 0, [1, 1], list(range(0, 64, 2)) + [1] * 9, 300),
    ([130], 2, 4, 4, 256, 128, "bf16", 20.0, 33, [0], [2, 4, -1, 1], 1),
    ([70, 300], 2, 40, 2, 128, 16, "e4m3", 0, 0, [1, 0], list(range(40)), 0),      # 20 rows a key head
    ([70], 3, 24, 1, 256, 32, "bf16", 0, 0, [2], list(range(24))[::-1], 0),
    ([130], 1, 17, 1, 64, 16, "e4m3", 0, 60, [0], list(range(17)), 0),
    ([40, 7], 2, 6, 3, 64, 16, "bf16", 0, 0, [1, 0], [r * 5 % 8 - 1 for r in range(700)], 0),   # past the list in LDS
    (list(range(1, 301)), 2, 4, 2, 64, 16, "bf16", 0, 0, [b % 4 - 1 for b in range(300)], [3, 0], 0),
]


@pytest.mark.parametrize("lens,n,Hq,heads,D,page,dtype,softcap,window,row,chosen,short", ROWS)
def test_rows(lens, n, Hq, heads, D, page, dtype, softcap, window, row, chosen, short):
    c = Case(lens, n, Hq, heads, D, page, E4M3 if dtype == "e4m3" else torch.bfloat16, seed=D + n)
    say("rows", lens, n, Hq, heads, D, page, dtype, softcap, window, row, chosen)
    B, R = len(lens), len(chosen)
    _, L = c.attend(softcap, window)
    keys = max(lens) + n - short
    wide = torch.full((B, R + 1, keys + 3), 7.0, device=dev())
    attn = wide[:, :R, 1:1 + keys]
    pld.pld_cache_attn_rows(c.q, c.k, c.t, c.d_lens, d_i32(row), d_i32(chosen), L, attn,
                            k_scale=c.ks, softcap=softcap, window=window)
    got, lse = f64(wide), f64(L)
    assert (got[:, R] == 7).all() and (got[:, :, 0] == 7).all() and (got[:, :, keys + 1:] == 7).all()
    got = got[:, :R, 1:1 + keys]
    for b in range(B):
        pos = lens[b] - 1 + row[b]
        if not 0 <= row[b] < n:
            assert (got[b] == 7).all()
            continue
        end = min(pos + 1, keys)
        assert (got[b, :, end:] == 7).all()
        for r, h in enumerate(chosen):
            if not 0 <= h < Hq:
                assert np.isnan(got[b, r, :end]).all()
                continue
            kv = h // (Hq // heads)
            k = ref.cache_rows(c.k, c.ks, c.table, b, kv, pos + 1)
            w, _, x, tol, _ = ref.attn_row(f64(c.q[b, row[b], h]), k, k, pos, D ** -0.5, softcap, window)
            w = w * np.exp(x - lse[b, row[b], h])          # from the log sum that the call was given
            # the score's and the difference's errors in the exponent, the exponential's own
            rel = np.expm1(2 * tol + 16 * U * (1 + abs(x) + np.abs(np.log(np.maximum(w, 1e-38)))))
            off = np.abs(got[b, r, :end] - w[:end]) - rel[:end] * w[:end]
            assert off.max() <= 2.0 ** -126, (b, r, off.max())
            if window:
                assert (got[b, r, :max(0, min(end, pos + 1 - window))] == 0).all()


def test_rows_bad_pages_and_ends():
    c = Case([100, 100, 0], 2, 4, 2, 64, 16, seed=2)
    _, L = c.attend()
    c.table[0, 1] = -3
    attn = torch.full((3, 2, 140), 7.0, device=dev())
    # sequence 1 claims a position past its table (7 pages: 112 positions)
    c.lens = [100, 130, 0]
    pld.pld_cache_attn_rows(c.q, c.k, d_i32(c.table), d_i32(c.lens), d_i32([1, 1, 0]), d_i32([0, 3]), L, attn)
    a = attn.cpu().numpy()
    assert np.isnan(a[0, :, 16:32]).all() and not np.isnan(a[0, :, :16]).any()
    assert not np.isnan(a[0, :, 32:]).any() and (a[0, :, 101:] == 7).all()
    cap = c.table.shape[1] * 16
    assert not np.isnan(a[1, :, :cap]).any() and np.isnan(a[1, :, cap:131]).all() and (a[1, :, 131:] == 7).all()
    assert (a[2] == 7).all()


# ------------------------------------------------------------------ log probabilities
LOGPROBS = [
    # B, n, V, type, tau, top, kind
    (1, 1, 1, "f32", 1.0, 1, "normal"),
    (2, 3, 7, "bf16", 1.0, 10, "normal"),
    (3, 2, 64, "f32", 0.5, 64, "ties"),
    (2, 4, 1001, "bf16", 2.0, 5, "ties"),
    (4, 11, 32000, "f32", 1.0, 5, "normal"),
    (2, 17, 50001, "bf16", 0.8, 20, "normal"),
    (2, 3, 4096, "bf16", 1.0, 64, "equal"),
    (2, 3, 9000, "f32", 1.0, 64, "equal"),
    (2, 5, 128256, "bf16", 1.0, 20, "masked"),
    (3, 4, 5000, "f32", 0.7, 12, "masked"),
    (2, 3, 3001, "f32", 0.05, 8, "lowest"),
    (2, 3, 12345, "bf16", 1.0, 30, "sorted"),
    (1, 2, 1000003, "bf16", 1.0, 0, "normal"),
    (1, 3, 40000, "f32", 1.0, 33, "block"),
    (1, 2, 200003, "f32", 1.0, 64, "ties"),        # a row's maxima in several rounds
    (2, 3, 140001, "bf16", 1.5, 64, "masked"),
    (1, 2, 262144, "bf16", 1.0, 40, "equal"),
    (1, 2, 160001, "f32", 1.0, 64, "normal"),
    (2, 2, 128256, "bf16", 1.0, 64, "normal"),
    (1, 2, 100000, "f32", 1.0, 33, "block"),       # most of the best side by side
    (1, 2, 100000, "f32", 1.0, 64, "sorted1"),
    (700, 2, 129, "bf16", 1.0, 3, "normal"),       # more sequences than threads of a block
]


@pytest.mark.parametrize("B,n,V,dtype,tau,top,kind", LOGPROBS)
def test_token_logprobs(B, n, V, dtype, tau, top, kind):
    say("logprobs", B, n, V, dtype, tau, top, kind)
    rng = np.random.default_rng(V + n)
    z = rng.standard_normal((B, n, V), dtype=np.float32) * 3
    if kind == "ties":
        z = np.round(z)                            # signed zeros among them
    elif kind == "equal":
        z[:] = -1.5
        z[0, 0, V // 2:] = 0.0
        z[0, 0, V // 2 + 1::2] = -0.0
    elif kind == "masked":
        z[:, :, rng.random(V) < 0.97] = -np.inf
        z[0, 0] = -np.inf                          # nothing is left
        z[0, 1] = -np.inf
        z[0, 1, V - 2] = 3.0                       # one token is
    elif kind == "lowest":
        z[:, :, rng.random(V) < 0.5] = torch.finfo(torch.float32).min
        z[0, 0] = torch.finfo(torch.float32).min
    elif kind == "sorted":
        z[0] = np.sort(z[0], -1)                   # the largest last
        z[1] = np.sort(z[1], -1)[:, ::-1]
    elif kind == "sorted1":
        z[0, 0], z[0, 1] = np.sort(z[0, 0]), np.sort(z[0, 1])[::-1]
    elif kind == "block":
        z[:, :, 1000:1600] += 20                   # all the large ones side by side
    Z = torch.from_numpy(z).to(torch.float32 if dtype == "f32" else torch.bfloat16).to(dev())
    # odd offsets: rows start off a 16-byte boundary
    wide = torch.full((B, n + 1, V + 3), 50.0, dtype=Z.dtype, device=dev())
    wide[:, :n, 1:V + 1] = Z
    tokens = rng.integers(0, V, (B, n)).astype(np.int32)
    tokens[0, 0] = V if V > 1 else 0
    tokens[-1, -1] = -1
    count = np.full(B, n, np.int32)
    count[-1] = n - 1 if n > 2 else n
    if B > 2:
        count[1] = n + 1                           # counts as 0
    results = []
    for src in (Z, wide[:, :n, 1:V + 1]):
        lp = torch.full((B, n), 7.0, device=dev())
        ent = torch.full((B, n), 7.0, device=dev())
        ids = torch.full((B, n, top), -7, dtype=torch.int32, device=dev()) if top else None
        tlp = torch.full((B, n, top), 7.0, device=dev()) if top else None
        need = pld.pld_token_logprobs_workspace_bytes(B, n, V, pld.PLD_F32 if dtype == "f32" else pld.PLD_BF16, top)
        ws = torch.full((need,), 0x7f, dtype=torch.uint8, device=dev())
        pld.pld_token_logprobs(src, d_i32(tokens), lp, ws, count=d_i32(count), temperature=tau,
                               entropy=ent, top_ids=ids, top_logprobs=tlp)
        results.append([x if x is None else x.cpu().numpy() for x in (lp, ent, ids, tlp)])
        bare = torch.full((B, n), 7.0, device=dev())
        pld.pld_token_logprobs(src, d_i32(tokens), bare, ws, count=d_i32(count), temperature=tau)
        assert np.array_equal(bare.cpu().numpy(), results[-1][0], equal_nan=True)
    zz = f64(Z)
    for lp, ent, ids, tlp in results:
        for b in range(B):
            cnt = int(count[b]) if 0 <= count[b] <= n else 0
            assert (lp[b, cnt:] == 7).all() and (ent[b, cnt:] == 7).all()
            assert not top or ((ids[b, cnt:] == -7).all() and (tlp[b, cnt:] == 7).all())
            for i in range(cnt):
                want, H, order = ref.logprob_row(zz[b, i], tau)
                # a lane's share of the sum and the tree over lanes, blocks and segments; the
                # exponentials; the quotient by the temperature
                add = (V / 64 + 96) * U
                near = lambda x, y: x == y or abs(x - y) <= add + 8 * U * (abs(y) + 1) or \
                    (y < -1e37 and x < -1e37)
                t = tokens[b, i]
                if 0 <= t < V:
                    assert near(lp[b, i], want[t]), (b, i, lp[b, i], want[t])
                else:
                    assert np.isnan(lp[b, i])
                assert abs(ent[b, i] - H) <= 2 * add * (1 + H) + 16 * U * (1 + H), (b, i, ent[b, i], H)
                if top:
                    k = min(top, V)
                    assert np.array_equal(ids[b, i, :k], order[:k]), (b, i, ids[b, i], order[:k])
                    assert (ids[b, i, k:] == -1).all() and (tlp[b, i, k:] == -np.inf).all()
                    assert all(near(x, want[o]) for x, o in zip(tlp[b, i, :k], order)), (b, i)


# ------------------------------------------------------------------ refusals
def test_binding_refusals():
    """Wrong types, shapes, devices and strides are refused before anything is enqueued."""
    c = Case([20], 2, 4, 2, 64, 16, seed=1)
    out = torch.empty_like(c.q)
    ws = torch.zeros(pld.pld_cache_attn_workspace_bytes(1, 2, 4, 2, 64), dtype=torch.uint8, device=dev())
    good = dict(q=c.q, k_cache=c.k, v_cache=c.v, table=c.t, lens=c.d_lens, out=out, workspace=ws)
    pld.pld_cache_attn(**good)
    q8 = c.k.float().to(E4M3)
    for bad in (dict(q=c.q.float()), dict(q=c.q[:, :, :, :32]), dict(q=c.q.cpu()), dict(lens=c.d_lens.long()),
                dict(lens=c.d_lens.repeat(2)), dict(table=c.t.long()), dict(table=c.t.repeat(2, 1)),
                dict(v_cache=c.v[:1]), dict(k_cache=q8, v_cache=q8), dict(k_scale=torch.zeros(1, device=dev())),
                dict(lse=torch.zeros(1, 2, 3, device=dev())), dict(out=out.transpose(2, 3)),
                dict(draft_len=torch.zeros(2, dtype=torch.int32, device=dev())), dict(v_cache=c.v.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(TypeError):
            pld.pld_cache_attn(**{**good, **bad})
    for bad, status in ((dict(scale=0.0), 1), (dict(scale=math.inf), 1), (dict(softcap=-1.0), 1),
                        (dict(window=-1), 1), (dict(workspace=ws[:-256] if ws.numel() > 256 else ws[:16]), 3)):
        with pytest.raises(pld.PLDError) as e:
            pld.pld_cache_attn(**{**good, **bad})
        assert e.value.status == status, bad
    with pytest.raises(TypeError):
        pld.pld_cache_attn_rows(c.q, c.k, c.t, c.d_lens, d_i32([0]), d_i32([0, 1]), torch.zeros(1, 2, 4, device=dev()),
                                torch.zeros(1, 3, 30, device=dev()))
    with pytest.raises(TypeError):
        pld.pld_cache_write(c.q, c.q, c.q, c.k, c.v, c.t, c.d_lens, out)          # 4 key heads for 2
    z = torch.zeros(1, 2, 100, device=dev())
    need = pld.pld_token_logprobs_workspace_bytes(1, 2, 100, pld.PLD_F32, 3)
    good = dict(logits=z, tokens=d_i32([[1, 2]]), logprob=torch.zeros(1, 2, device=dev()),
                workspace=torch.zeros(need, dtype=torch.uint8, device=dev()))
    ids, tl = torch.zeros(1, 2, 3, dtype=torch.int32, device=dev()), torch.zeros(1, 2, 3, device=dev())
    pld.pld_token_logprobs(**good, top_ids=ids, top_logprobs=tl)
    for bad in (dict(logits=z.half()), dict(tokens=d_i32([[1, 2, 3]])), dict(top_ids=ids), dict(top_ids=ids, top_logprobs=tl[:, :, :2])):
        with pytest.raises(TypeError):
            pld.pld_token_logprobs(**{**good, **bad})
    for bad in (dict(temperature=0.0), dict(temperature=math.nan), dict(temperature=-1.0)):
        with pytest.raises(pld.PLDError) as e:
            pld.pld_token_logprobs(**{**good, **bad})
        assert e.value.status == 1


# ------------------------------------------------------------------ together
class TinyModel:
    """One attention layer over a copy task: embeddings, heads, and logits that favour the
    token after the one that the attention copies.  Weights are random; what is checked is
    that every call's results are those of its plain form on the same inputs."""

    def __init__(self, B, max_len, V, K, dtype, seed=0):
        rng = np.random.default_rng(seed)
        self.Hq, self.heads, self.D, self.V, self.K = 8, 2, 64, V, K
        # every token's query, keys and values
        self.qkv = normal(rng, V, (self.Hq + 2 * self.heads) * self.D)
        self.wo = normal(rng, self.Hq * self.D, V, gain=0.2)
        self.qn, self.kn = normal(rng, self.D, gain=0.1) + 1, normal(rng, self.D, gain=0.1) + 1
        angle = np.arange(max_len + K + 1)[:, None] * 10000.0 ** (-np.arange(0, self.D, 2) / self.D)
        self.rope = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], -1).astype(np.float32)).to(dev())
        self.cache = PagedCache(B, max_len + K + 1, self.heads, self.D, page_size=16, dtype=dtype)
        self.cache.table.copy_(torch.from_numpy(rng.permutation(self.cache.table.numel()).astype(np.int32)).view_as(self.cache.table))
        n = K + 1
        self.q = torch.zeros((B, n, self.Hq, self.D), dtype=torch.bfloat16, device=dev())
        self.out = torch.zeros_like(self.q)
        self.lse = torch.zeros((B, n, self.Hq), device=dev())
        self.logits = torch.zeros((B, n, V), device=dev())
        self.cache.reserve(n, self.Hq)

    def rows(self, tokens, lens, draft_len):
        """tokens [B][n]: the rows' own tokens."""
        Hq, H, D = self.Hq, self.heads, self.D
        x = self.qkv[tokens.long()]
        q, k, v = (t.unflatten(-1, (-1, D)) for t in x.split([Hq * D, H * D, H * D], -1))
        n = tokens.shape[1]
        if n != self.q.shape[1]:
            q_out, out, lse = (torch.zeros((x.shape[0], n) + t.shape[2:], dtype=t.dtype, device=dev())
                               for t in (self.q, self.out, self.lse))
        else:
            q_out, out, lse = self.q, self.out, self.lse
        self.cache.write(q, k, v, lens, q_out, draft_len=draft_len, q_norm=self.qn, k_norm=self.kn, rope=self.rope)
        self.cache.attend(q_out, lens, out, draft_len=draft_len, lse=lse)
        return out

    def step(self, step, lens):
        last = torch.gather(self.tokens, 1, (lens.long() - 1)[:, None])
        rows = torch.cat([last, step.draft.clamp(min=0)], 1)
        out = self.rows(rows, lens, step.draft_len)
        self.logits.copy_(out.flatten(2).float() @ self.wo.float())
        return self.logits


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("capture", [False, True])
def test_loop_with_cache_and_logprobs(dtype, capture):
    """A generation loop whose drafts are ranked by the attention rows that the cache gives:
    prompt in chunks, then draft, write, attend, verify, log probabilities, artifact and
    commit.  Every token it emits is the best one of the finished sequence read again in
    chunks through a cache of its own, up to the roundings of the two attentions; log
    probabilities and artifact rows are those of the plain forms.  The captured form replays
    one step as a graph, other work between the replays."""
    B, K, V, prompt, more = 3, 6, 50, [40, 57, 23], 24
    max_len = max(prompt) + more + 2 * K
    rng = np.random.default_rng(1)
    toks = np.zeros((B, max_len), np.int32)
    base = rng.integers(0, V, 12)
    for b in range(B):
        toks[b, :prompt[b]] = np.resize(base, prompt[b])
    limit = d_i32([p + more for p in prompt])

    def fill(model, tokens, lens):
        """The prompts but their last token into the cache, 16 rows at a time."""
        for s in range(0, max(prompt), 16):
            rows = torch.zeros((B, 16), dtype=torch.int32, device=dev())
            cnt = []
            for b in range(B):
                m = max(0, min(16, prompt[b] - 1 - s))
                rows[b, :m] = tokens[b, s:s + m]
                cnt.append(m - 1)
            model.rows(rows, d_i32([s + 1] * B), d_i32(cnt))

    model = TinyModel(B, max_len, V, K, dtype)
    tokens, lens = d_i32(toks), d_i32(prompt)
    model.tokens = tokens
    fill(model, tokens, lens)
    heads = d_i32([1, 6, 3])
    attn = torch.zeros((B, 3, max_len), device=dev())
    attn[:, :, 5] = 1.0
    step = DraftStep(B, max_len, K, mode="fused")
    step.set_logprobs(V, bf16=False, top=4)
    seen = []

    def refresh(step, lens):
        model.cache.weights(model.q, lens, step.accept_len, heads, model.lse, attn)
        if not capture:
            seen.append([t.clone() for t in (lens, step.accept_len, step.out_tokens, step.out_count, step.logprob,
                                             step.top_ids, model.logits, attn, model.q, model.lse)])

    if not capture:
        steps = decode_loop(step, tokens, lens, limit, model.step, attn=attn, refresh=refresh, check_every=1)
        say("steps", steps, "for", more, "tokens")
    else:
        side = torch.cuda.Stream()
        keep = [t.clone() for t in (tokens, lens, attn)]

        def one():
            step.make_draft(tokens, lens, attn=attn)
            step.verify(model.step(step, lens))
            refresh(step, lens)
            step.commit(tokens, lens, limit=limit)

        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            one()                                  # warm-up; its effects are taken back
        torch.cuda.current_stream().wait_stream(side)
        for t, old in zip((tokens, lens, attn), keep):
            t.copy_(old)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            one()
        noise = torch.zeros(1000, device=dev())
        for _ in range(more + 2):
            graph.replay()
            noise += 1
            torch.cuda.synchronize()
            if bool((lens >= limit).all()):
                break
    got = tokens.cpu().numpy()
    again, n = TinyModel(B, max_len, V, K, dtype), 16
    wo = f64(again.wo)
    for s in range(0, max(prompt) + more, n):
        rows = np.zeros((B, n), np.int32)
        cnt = [max(0, min(n, prompt[b] + more - 1 - s)) for b in range(B)]
        for b in range(B):
            rows[b, :cnt[b]] = got[b, s:s + cnt[b]]
        out = f64(again.rows(d_i32(rows), d_i32([s + 1] * B), d_i32([m - 1 for m in cnt])))
        for b in range(B):
            for i in range(cnt[b]):
                t = s + i + 1
                if t >= prompt[b]:
                    o = out[b, i].reshape(-1)
                    z, size = o @ wo, np.abs(o) @ np.abs(wo)
                    # both outputs are off by at most out_bound, twice a bf16 half step of
                    # sums that are at most a few times the outputs here
                    assert z[got[b, t]] >= z.max() - 8 * 2.0 ** -8 * size.max(), (b, t, z[got[b, t]], z.max())
    for lens0, acc, out_t, out_c, lp, ids, z, a, q, lse in seen[:6]:
        zz, L0, acc = f64(z), lens0.cpu().numpy(), acc.cpu().numpy()
        for b in range(B):
            for i in range(int(out_c[b])):
                w, _, order = ref.logprob_row(zz[b, i], 1.0)
                assert abs(float(lp[b, i]) - w[int(out_t[b, i])]) <= 1e-5 * (1 + abs(w[int(out_t[b, i])]))
                assert ids[b, i].tolist() == order[:4].tolist()
            pos = int(L0[b]) - 1 + int(acc[b])
            for r, h in enumerate((1, 6, 3)):
                k = ref.cache_rows(model.cache.k, model.cache.k_scale, model.cache.table.cpu().numpy(), b, h // 4, pos + 1)
                w, _, _, tol, _ = ref.attn_row(f64(q[b, acc[b], h]), k, k, pos, 0.125, 0.0, 0)
                assert abs(f64(a[b, r, :pos + 1]) - w).max() <= 1e-5, (b, r)
                assert abs(f64(a[b, r, :pos + 1]).sum() - 1) <= 1e-4


def test_two_streams_at_once():
    """Two callers with their own workspaces on streams of their own, one of them over the
    other's cache: the results are those of the calls alone."""
    a = Case([5000, 3, 900], 5, 8, 2, 128, 16, seed=1)
    b = Case([2000, 60], 3, 16, 4, 64, 32, E4M3, seed=2)
    wa, wb = a.attend(), b.attend(softcap=20.0)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(10):
        with torch.cuda.stream(sa):
            x = a.attend()
        with torch.cuda.stream(sb):
            y = b.attend(softcap=20.0)
        got.append((x, y))
    torch.cuda.synchronize()
    for x, y in got:
        assert np.array_equal(bits(x[0]), bits(wa[0])) and np.array_equal(bits(x[1]), bits(wa[1]))
        assert np.array_equal(bits(y[0]), bits(wb[0])) and np.array_equal(bits(y[1]), bits(wb[1]))


def test_a_workspace_that_grew_stays_with_its_calls():
    """A prepared call keeps its workspace when the cache's grows: memory that is allocated
    afterwards is left alone, and the call's results stay the same."""
    rng = np.random.default_rng(8)
    cache = PagedCache(2, 2000, 2, 64, page_size=16)
    cache.k.copy_(normal(rng, *cache.k.shape))
    cache.v.copy_(normal(rng, *cache.v.shape))
    q, lens = normal(rng, 2, 1, 8, 64), d_i32([1990, 700])
    out = torch.zeros_like(q)
    call = cache.attend(q, lens, out, prepare=True)
    call()
    want, size = out.clone(), cache.workspace.numel()
    cache.attend(normal(rng, 2, 9, 8, 64), d_i32([1900, 60]), torch.zeros((2, 9, 8, 64), dtype=torch.bfloat16, device=dev()))
    assert cache.workspace.numel() > size
    later = [torch.full((size,), 0x55, dtype=torch.uint8, device=dev()) for _ in range(4)]
    out.zero_()
    call()
    assert np.array_equal(bits(out), bits(want)) and all(bool((t == 0x55).all()) for t in later)


def test_two_graphs_share_a_workspace():
    """An attention and log probabilities captured twice over one workspace each, replayed in
    turn with the program's own work between: every replay is the eager call's result."""
    a = Case([5000, 3, 900], 5, 8, 2, 128, 16, seed=1)
    b = Case([40, 2000], 9, 16, 2, 64, 32, seed=2)
    ws = torch.zeros(max(pld.pld_cache_attn_workspace_bytes(len(c.lens), c.n, c.Hq, c.heads, c.D) for c in (a, b)),
                     dtype=torch.uint8, device=dev())
    rng = np.random.default_rng(3)
    z = [torch.from_numpy(rng.standard_normal((2, 3, V), dtype=np.float32)).to(dev()) for V in (5000, 33000)]
    lws = torch.zeros(pld.pld_token_logprobs_workspace_bytes(2, 3, 33000, pld.PLD_F32, 7), dtype=torch.uint8, device=dev())
    tok = d_i32(np.full((2, 3), 4))
    runs = []
    for c, x in zip((a, b), z):
        out, L = torch.zeros_like(c.q), torch.zeros((len(c.lens), c.n, c.Hq), device=dev())
        lp, ids = torch.zeros((2, 3), device=dev()), torch.zeros((2, 3, 7), dtype=torch.int32, device=dev())
        tl = torch.zeros((2, 3, 7), device=dev())

        def run(c=c, x=x, out=out, L=L, lp=lp, ids=ids, tl=tl):
            pld.pld_cache_attn(c.q, c.k, c.v, c.t, c.d_lens, out, ws, lse=L)
            pld.pld_token_logprobs(x, tok, lp, lws, top_ids=ids, top_logprobs=tl)

        run()
        outs = (out, L, lp, ids, tl)
        want = [bits(t) for t in outs]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        runs.append((graph, outs, want))
    noise = torch.zeros(1000, device=dev())
    for turn in range(6):
        for graph, outs, want in runs:
            for t in outs:
                t.zero_()
            graph.replay()
            noise += 1
            if turn % 2:
                torch.cuda.synchronize()
            assert all(np.array_equal(bits(t), w) for t, w in zip(outs, want)), turn


@pytest.mark.parametrize("sample", [False, True])
def test_plans_and_verification_give_log_probabilities(sample):
    """After set_logprobs, verify() and a prepared plan both leave the emitted tokens' log
    probabilities, those of pld_token_logprobs alone; without it they leave none."""
    B, K, V, T = 3, 4, 1000, 200
    rng = np.random.default_rng(2)
    tokens, lens = d_i32(rng.integers(0, 30, (B, T + K + 1))), d_i32([T, 150, 90])
    attn = torch.from_numpy(rng.random((B, 2, T + K + 1), dtype=np.float32)).to(dev())
    z = torch.from_numpy(rng.standard_normal((B, K + 1, V), dtype=np.float32) * 3).to(dev())
    step = DraftStep(B, T + K + 1, K, mode="fused")
    if sample:
        step.set_sampling(0.7, V, False, torch.from_numpy(rng.random((B, K + 1), dtype=np.float32)).to(dev()))
    step.set_logprobs(V, bf16=False, top=5, temperature=0.7)
    step.logprob.fill_(7.0)
    step.make_draft(tokens, lens, attn=attn)
    step.verify(z)
    want = torch.full_like(step.logprob, 7.0)
    ent, ids = torch.zeros_like(want), torch.zeros_like(step.top_ids)
    tl = torch.zeros_like(step.top_logprobs)
    pld.pld_token_logprobs(z, step.out_tokens, want, step.logprob_ws, count=step.out_count, temperature=0.7, entropy=ent,
                           top_ids=ids, top_logprobs=tl)
    assert np.array_equal(bits(step.logprob), bits(want))
    for b in range(B):
        m = int(step.out_count[b])
        assert m >= 1 and not (step.logprob[b, :m] == 7).any() and (step.logprob[b, m:] == 7).all()
        assert np.array_equal(bits(step.top_ids[b, :m]), bits(ids[b, :m]))
        assert np.array_equal(bits(step.logprob_entropy[b, :m]), bits(ent[b, :m]))
        assert np.array_equal(bits(step.top_logprobs[b, :m]), bits(tl[b, :m]))
    ops = step.plan(tokens, lens, z, attn=attn)
    assert [name for name, _ in ops][-1] == "token_logprobs"
    step.logprob.fill_(7.0)
    for _, op in ops:
        op()
    assert np.array_equal(bits(step.logprob), bits(want))
    step.set_logprobs(None, False)
    assert "token_logprobs" not in [name for name, _ in step.plan(tokens, lens, z, attn=attn)]
    step.verify(z)
