"""A prompt's pass against plain references (prompt_ref.py): packed attention, the packed write with
positions on several axes, the pages of a pool, and a run of them with the cache's calls."""
import math

import numpy as np
import pytest
import torch

import model_ref as ref
import paper_2412_01447_amd as pld
import prompt_ref
from gpu_helpers import d_i32, dev, random_plan, say
from model_ref import U, f64
from paper_2412_01447_amd.cache import PagedCache, PagePool

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn
NAN, INF = math.nan, math.inf


def normal(rng, *shape, gain=1.0):
    x = rng.standard_normal(shape, dtype=np.float32) * gain
    return torch.from_numpy(x).to(torch.bfloat16).to(dev())


def bits(t):
    t = t.contiguous()
    return t.view(torch.uint8).cpu().numpy() if t.dtype == E4M3 else \
        t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).cpu().numpy()


def starts_of(lens, at=0):
    return [at] + [at + int(x) for x in np.cumsum(lens)]


# ------------------------------------------------------------------ attention
class Prompt:
    """Packed rows of sequences of `lens`, `at` rows before them and `pad` behind."""

    def __init__(self, lens, Hq, heads, D, at=0, pad=0, seed=0, gain=2.0, split=False):
        rng = np.random.default_rng(seed)
        self.starts = starts_of(lens, at)
        N = self.N = max(1, self.starts[-1] + pad)
        if split:                    # one projection's output
            q, k, v = normal(rng, N, (Hq + 2 * heads) * D).split([Hq * D, heads * D, heads * D], -1)
            self.q, self.k, self.v = q.unflatten(-1, (Hq, D)), k.unflatten(-1, (heads, D)), v.unflatten(-1, (heads, D))
            q.mul_(gain)
        else:
            self.q, self.k, self.v = normal(rng, N, Hq, D, gain=gain), normal(rng, N, heads, D), normal(rng, N, heads, D)
        self.d_starts = d_i32(self.starts)

    def attend(self, lse=True, out=None, **kw):
        o = torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device=dev()) if out is None else out
        L = torch.full(self.q.shape[:2], 7.0, device=dev()) if lse else None
        pld.pld_prompt_attn(self.q, self.k, self.v, self.d_starts, o, lse=L, **kw)
        return o, L

    def check(self, rows=None, poisoned=(), **kw):
        o, L = self.attend(**kw)
        return prompt_ref.check_attn(self.q, self.k, self.v, self.starts, o, L, rows=rows, poisoned=poisoned, **kw)


ATTN = [
    # lens, Hq, heads, D, rows before, rows behind, softcap, window
    ([1], 1, 1, 128, 0, 0, 0, 0),
    ([1, 1, 1], 4, 2, 64, 0, 0, 0, 0),
    ([2, 0, 3, 0, 0, 1], 8, 8, 128, 3, 5, 0, 0),
    ([63, 64, 65], 4, 1, 128, 0, 0, 0, 0),
    ([31, 33, 1, 127, 129], 6, 2, 64, 1, 2, 0, 0),
    ([130], 7, 1, 128, 0, 70, 0, 0),
    ([257, 5], 5, 5, 128, 7, 0, 0, 0),
    ([100, 28], 12, 1, 256, 0, 1, 0, 0),
    ([66, 90], 2, 2, 256, 5, 9, 0, 0),
    ([300], 2, 1, 64, 0, 0, 0, 0),
    ([150, 40], 4, 2, 128, 0, 0, 30.0, 0),
    ([150, 40], 4, 2, 64, 0, 3, 2.0, 0),
    ([70, 40], 4, 2, 256, 0, 3, 5.0, 17),
    ([200, 90], 4, 2, 128, 2, 0, 0, 1),
    ([200, 90], 4, 2, 64, 0, 0, 0, 37),
    ([400], 2, 1, 128, 0, 0, 0, 64),
    ([333], 3, 1, 128, 0, 0, 50.0, 200),
]


@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attn(case):
    lens, Hq, heads, D, at, pad, cap, window = ATTN[case]
    p = Prompt(lens, Hq, heads, D, at, pad, seed=case, split=case % 2 == 1)
    assert p.check(softcap=float(cap), window=window) == sum(lens) * Hq


@pytest.mark.parametrize("D,Hq,heads", [(64, 24, 4), (128, 32, 8), (256, 4, 2)])
def test_attn_long(D, Hq, heads):
    """Some thousand rows: blocks that see many tiles, checked at rows around the tiles' ends."""
    lens = [2100, 1, 700, 63]
    p = Prompt(lens, Hq, heads, D, 0, 11, seed=5)
    rows = {0, 1, 63, 64, 65, 127, 128, 255, 256, 257, 1023, 1500, 2047, 2048, 2099, 2100, 2101, 2164, 2500, 2800, 2801, 2863}
    assert p.check(rows=rows) == len(rows) * Hq
    assert p.check(rows=rows, window=1000, softcap=20.0) == len(rows) * Hq


def test_attn_long_of_narrow_heads():
    """Heads of 64 where a wave has 64 rows: the ends of tiles and sequences, a window, what is not finite."""
    p = Prompt([5000, 1101], 48, 8, 64, 3, 11, seed=6)
    rows = {0, 3, 4, 66, 67, 68, 130, 131, 1026, 3000, 4999, 5002, 5003, 5004, 5066, 5067, 6000, 6102, 6103, 6113}
    assert p.check(rows=rows) == (len(rows) - 2) * 48
    a, la = p.attend(window=1000)
    assert p.check(rows=rows, window=1000) == (len(rows) - 2) * 48
    p.v[1], p.k[2], p.v[500], p.k[6105] = INF, NAN, NAN, INF
    b, lb = p.attend(window=1000)
    seen = torch.ones(p.N, dtype=torch.bool, device=dev())
    seen[500:1500] = False                          # (rows that see the NaN)
    assert torch.equal(a[seen], b[seen]) and torch.equal(la[seen], lb[seen]) and b[500:1500].isnan().all()


def test_attn_random_shapes():
    rng, iters = random_plan(11, 24)
    for it in range(iters):
        D = int(rng.choice([64, 128, 256]))
        heads, G = int(rng.choice([1, 2, 3, 4])), int(rng.choice([1, 2, 3, 4, 5, 7, 8, 12]))
        lens = [int(x) for x in rng.integers(0, int(rng.choice([2, 40, 300])), int(rng.integers(1, 9)))]
        if sum(lens) == 0:
            continue
        cap, window = float(rng.choice([0, 0, 4.0, 50.0])), int(rng.choice([0, 0, 1, 5, 100]))
        say("attn", it, lens, D, heads, G, cap, window)
        p = Prompt(lens, heads * G, heads, D, int(rng.integers(0, 70)), int(rng.integers(0, 70)), seed=100 + it, split=bool(it % 2))
        rows = set(int(x) for x in rng.integers(0, p.N, 24))
        p.check(rows=rows, softcap=cap, window=window)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 50])
def test_attn_unseen_rows_do_not_matter(D, window):
    """NaN, infinities and the largest numbers in rows of other sequences, before the window, behind a
    row and behind the last sequence: rows that do not see them are as without them; those that do
    see them are NaN, or what the formula gives."""
    lens = [90, 150, 40]
    bad = {10: INF, 89: NAN, 95: -INF, 170: NAN, 239: INF, 241: NAN, 282: NAN, 283: INF}
    clean = Prompt(lens, 4, 2, D, 0, 5, seed=3)
    o, L = clean.attend(window=window)
    for which in ("v", "k", "both"):
        p = Prompt(lens, 4, 2, D, 0, 5, seed=3)
        for r, x in bad.items():
            if which != "v":
                p.k[r] = x
            if which != "k":
                p.v[r, :, r % D] = x
        assert p.check(window=window, poisoned=set(bad)) > 0
        o2, L2 = p.attend(window=window)
        b = bits(o2) != bits(o)
        for a, e in prompt_ref.sequences(p.starts, p.N):
            for r in range(a, e):
                seen = [x for x in bad if (max(a, r + 1 - window) if window else a) <= x <= r]
                if not seen:
                    assert not b[r].any(), r
                elif which != "k":
                    assert np.isnan(f64(o2[r])).all(), r
                if seen and which != "k" and any(bad[x] != bad[x] for x in seen):
                    assert torch.isnan(L2[r]).all(), r


def test_attn_large_values():
    """Values of 2^89, and scores of some thousands: no weight or sum overflows."""
    p = Prompt([200], 2, 1, 128, seed=8)
    p.v.mul_(2.0 ** 86)
    p.q.mul_(100.0)
    o, L = p.attend()
    assert torch.isfinite(o).all() and torch.isfinite(L).all()
    rows = {0, 1, 64, 150, 199}
    prompt_ref.check_attn(p.q, p.k, p.v, p.starts, o, L, rows=rows)


def test_attn_falling_and_rising_scores():
    """Rows whose largest score comes first, last, or grows by more than the slack from tile to tile."""
    p = Prompt([400], 1, 1, 128, seed=4)
    for ramp in (torch.arange(400.0), 400 - torch.arange(400.0), (torch.arange(400.0) - 200).abs()):
        p.k.copy_((ramp * 0.5).to(dev())[:, None, None].expand(400, 1, 128) / 128)
        p.q.fill_(math.sqrt(128.0))
        p.check(rows={0, 63, 64, 65, 128, 200, 255, 256, 320, 399})


@pytest.mark.parametrize("D,B,cap", [(64, 1, 0), (64, 64, 0), (64, 1, 30.0), (128, 1, 0), (128, 300, 0), (128, 1, 30.0), (128, 300, 30.0),
                                     (256, 1, 0), (256, 1, 30.0)])
def test_attn_sums_of_equal_weights(D, B, cap):
    """A long sequence whose first keys score 5 below many equal ones: weights that are summed one by one round
    one way all along.  (Empty sequences behind it: the other block shapes.)"""
    N, first = 100000, 40
    p = Prompt([N] + [0] * (B - 1), 2, 1, D, seed=7)
    p.q.fill_(1.0)
    p.k.fill_(5 / math.sqrt(D))
    p.k[:first] = 0.0
    p.v.copy_(1 + torch.rand(p.v.shape, generator=torch.Generator(device=dev()).manual_seed(1), device=dev()))
    o, L = p.attend(softcap=float(cap))
    x = float(p.k[first, 0].double().sum()) * D ** -0.5
    tol = (D + 8) * U * x
    if cap:
        x, tol = cap * math.tanh(x / cap), tol + 16 * U * cap
    n = torch.arange(1, N + 1, dtype=torch.float64, device=dev())
    low, high = n.clamp(max=first), (n - first).clamp(min=0)
    total = low + high * math.exp(x)
    v = p.v[:, 0].double().cumsum(0)
    want = (v[:first][(low - 1).long()] + (v - v[first - 1]) * (high > 0)[:, None] * math.exp(x)) / total[:, None]
    lse = total.log()
    bound = tol + 8 * U * (lse.abs() + 1) + ((n + 1).log2() + 64) * 2 * U          # (model_ref.lse_bound)
    assert ((L.double() - lse[:, None]).abs() <= bound[:, None]).all(), (L.double() - lse[:, None]).abs().max()
    # model_ref.out_bound, and half a step of fp32 for each product of 16 keys
    bound = (2.0 ** -8 * 2.02 + 4 * tol + 2.0 ** -16 + n / 16 * U)[:, None, None] * want[:, None]
    assert ((o.double() - want[:, None]).abs() <= bound).all(), (o.double() / want[:, None] - 1).abs().max()


def test_attn_in_place_and_without_lse():
    a = Prompt([100, 60], 8, 2, 128, 1, 3, seed=2, split=True)
    o, L = a.attend()
    q = a.q.clone()
    kept = torch.cat([q[:1], q[161:]])
    a.attend(lse=False, out=a.q)
    assert (bits(a.q[1:161]) == bits(o[1:161])).all() and torch.equal(torch.cat([a.q[:1], a.q[161:]]), kept)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_attn_capped_scores_go_by_themselves(D):
    """Far scores beside a row's own, or unseen ones of the same tiles, do not change its bits."""
    p = Prompt([40, 100, 300], Hq=6, heads=2, D=D, seed=4)
    a, la = p.attend(softcap=30.0)
    p.q[140:] *= 40.0
    b, lb = p.attend(softcap=30.0)
    assert torch.equal(a[:140], b[:140]) and torch.equal(la[:140], lb[:140])
    p.k[100:140] *= 60.0                            # far for the rows that see them, not for those before
    c, lc = p.attend(softcap=30.0)
    assert torch.equal(a[:100], c[:100]) and torch.equal(la[:100], lc[:100]) and not torch.equal(a[100:140], c[100:140])
    p.check(softcap=30.0)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("sign,cap", [(1, 5.0), (-1, 0.5)])
def test_attn_infinite_capped_scores(D, sign, cap):
    """A key that makes scores infinite: the cap on either side, or NaN for the head as a whole."""
    p = Prompt([200], Hq=4, heads=2, D=D, seed=8)
    p.k[70, :, 3] = sign * INF
    o, L = p.attend(softcap=cap)
    q, k, v, o, L = f64(p.q), f64(p.k), f64(p.v), f64(o), L.cpu().numpy()
    met = 0
    for r in range(200):
        for h in range(4):
            s = cap * np.tanh(k[:r + 1, h // 2] @ q[r, h] * D ** -0.5 / cap)
            w = np.exp(s - s.max())
            want, size = w @ v[:r + 1, h // 2] / w.sum(), w @ np.abs(v[:r + 1, h // 2]) / w.sum()
            if r >= 70 and np.isnan(L[r, h]):
                assert np.isnan(o[r, h]).all()
                continue
            met += r >= 70
            # a weight's rounding, the output's, and the scores': (D + 8) 2^-24 of products whose sizes sum to 160 at most
            tol = (D + 8) * U * 160
            assert np.all(np.abs(o[r, h] - want) <= 2.0 ** -8 * (np.abs(want) + size) + 4 * tol * size)
            assert abs(L[r, h] - (np.log(w.sum()) + s.max())) <= 2 * tol + 1e-5
    say("infinite scores met", met)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("sign,cap", [(1, 5.0), (-1, 0.5)])
def test_attn_every_infinite_score_is_capped(D, sign, cap):
    """All rows that see a key which makes scores infinite of either sign: the cap's weight, and nothing of a mask's."""
    p = Prompt([200], Hq=4, heads=2, D=D, seed=8)
    p.k[70, :, 3] = sign * INF
    o, L = p.attend(softcap=cap)
    q, k, v, o, L = f64(p.q), f64(p.k), f64(p.v), f64(o), L.cpu().numpy()
    assert (q[70:, :, 3] != 0).all() and (q[70:, :, 3] > 0).any() and (q[70:, :, 3] < 0).any()
    met = 0
    for r in range(70, 200):
        for h in range(4):
            kk, vv = k[:r + 1, h // 2], v[:r + 1, h // 2]
            s = cap * np.tanh(kk @ q[r, h] * D ** -0.5 / cap)
            size = np.abs(np.delete(kk, 70, 0)) @ np.abs(q[r, h]) * D ** -0.5
            tol = (D + 8) * U * size.max() + 16 * U * cap
            want = s.max() + math.log(np.exp(s - s.max()).sum())
            w = np.exp(s - want)
            assert abs(L[r, h] - want) <= ref.lse_bound(tol, want, r + 1), (r, h, L[r, h], want)
            assert np.all(np.abs(o[r, h] - w @ vv) <= ref.out_bound(w @ vv, w @ np.abs(vv), tol)), (r, h)
            met += 1
    assert met == 130 * 4


@pytest.mark.parametrize("D,Hq,heads,lens,cap,window", [
    (64, 4, 2, [1, 31, 33, 64, 200], 30.0, 0), (128, 4, 2, [1, 31, 33, 64, 200], 30.0, 0), (256, 4, 2, [1, 31, 33, 64, 200], 30.0, 0),
    (128, 6, 2, [700], 0.5, 0), (64, 2, 1, [700], 5.0, 40), (128, 32, 8, [2300], 30.0, 0), (256, 4, 1, [900], 5.0, 300)])
def test_attn_capped_scores_of_minus_infinity(D, Hq, heads, lens, cap, window):
    """Finite queries and keys whose products pass fp32's range: scores of the cap, of either sign from head to head,
    where they are a row's first keys, all of a step, or all that it sees, as well."""
    p = Prompt(lens, Hq, heads, D, at=2, pad=3, seed=12)
    p.q[..., 0] = torch.tensor([-1.0, 1.0] * Hq)[:Hq].to(dev()) * 2.0 ** 65
    p.k[..., 0] = 0.0
    far = np.zeros(p.N, bool)
    for i, (a, b) in enumerate(prompt_ref.sequences(p.starts, p.N)):
        for lo, hi in ((0, 1 + 13 * i), (100, 170), (300, 650)):
            far[a + lo:min(b, a + hi)] = True
    p.k[torch.from_numpy(far).to(dev())] = 0.0
    p.k[torch.from_numpy(far).to(dev()), :, 0] = 2.0 ** 65
    o, L = p.attend(softcap=cap, window=window)
    q, k, v, o, L = f64(p.q), f64(p.k), f64(p.v), f64(o), L.cpu().numpy()
    near, met = {0, 1, 30, 31, 32, 33, 63, 64, 65, 100, 127, 128, 169, 170, 255, 256, 299, 300, 340, 649, 650}, 0
    for a, b in prompt_ref.sequences(p.starts, p.N):
        for r in range(a, b):
            if b - a > 300 and r - a not in near and r % 97:
                continue
            lo = max(a, r + 1 - window) if window else a
            for h in range(Hq):
                kk, vv = k[lo:r + 1, h // (Hq // heads)], v[lo:r + 1, h // (Hq // heads)]
                s = cap * np.tanh(kk @ q[r, h] * D ** -0.5 / cap)
                size = np.abs(kk[:, 1:]) @ np.abs(q[r, h, 1:]) * D ** -0.5
                tol = (D + 8) * U * size.max() + 16 * U * cap
                want = s.max() + math.log(np.exp(s - s.max()).sum())
                w = np.exp(s - want)
                assert abs(L[r, h] - want) <= ref.lse_bound(tol, want, r + 1 - lo), (r, h, L[r, h], want)
                assert np.all(np.abs(o[r, h] - w @ vv) <= ref.out_bound(w @ vv, w @ np.abs(vv), tol)), (r, h)
                met += far[lo:r + 1].any()
    assert met > 0


def test_attn_many_empty_sequences():
    lens = np.zeros(60000, int)
    lens[[0, 7, 30000, 30001, 59998]] = [5, 70, 1, 40, 3]
    p = Prompt(lens, 2, 1, 64, 2, 2, seed=6)
    want = Prompt([5, 70, 1, 40, 3], 2, 1, 64, 2, 2, seed=6)
    (o, L), (o2, L2) = p.attend(), want.attend()
    assert torch.equal(o, o2) and torch.equal(L, L2)
    want.check()


def test_attn_no_row_and_odd_starts():
    """No row at all; and starts that break the rule stay within the buffers."""
    p = Prompt([0, 0], 2, 1, 64, 0, 40, seed=6)
    o, L = p.attend()
    assert (o == 7).all() and (L == 7).all()
    for starts in ([5, 3, 40], [-7, 90, 2 ** 31 - 1], [2 ** 31 - 1, -5, 30], [40, 40, 40], [0, 2 ** 31 - 1, 40]):
        p.d_starts = d_i32(starts)
        p.attend()
    torch.cuda.synchronize()


def test_attn_far_rows():
    """Offsets past 2^31 elements: rows 2^16 elements apart."""
    N, S = 40000, 1 << 16
    big = torch.empty(N * S, dtype=torch.bfloat16, device=dev())
    rng = np.random.default_rng(1)
    p = Prompt([10], 2, 1, 64, seed=1)
    view = lambda at, heads: big.as_strided((N, heads, 64), (S, 64, 1), at)
    p.q, p.k, p.v, out = view(0, 2), view(256, 1), view(512, 1), view(1024, 2)
    for t in (p.q, p.k, p.v):
        t.copy_(normal(rng, *t.shape))
    out.fill_(7.0)
    p.starts = [0, 39000, 39900]
    p.N, p.d_starts = N, d_i32(p.starts)
    L = torch.full((N, 2), 7.0, device=dev())
    pld.pld_prompt_attn(p.q, p.k, p.v, p.d_starts, out, lse=L, window=300)
    rows = {0, 20000, 38999, 39000, 39001, 39500, 39899}
    assert prompt_ref.check_attn(p.q, p.k, p.v, p.starts, out, L, window=300, rows=rows) == 2 * len(rows)


def test_attn_captured_and_on_other_streams():
    """A captured call follows its starts; calls on two streams at once; replays between eager work."""
    p = Prompt([100, 60, 40], 8, 2, 128, seed=2)
    a = [p.attend() for _ in range(2)]
    assert torch.equal(a[0][0], a[1][0])
    g = torch.cuda.CUDAGraph()
    o, L = torch.zeros_like(p.q), torch.zeros(p.N, 8, device=dev())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        pld.pld_prompt_attn(p.q, p.k, p.v, p.d_starts, o, lse=L)
    for lens in ([200], [100, 60, 40], [1, 1, 198], [0, 150, 50]):
        p.starts = starts_of(lens)
        p.d_starts.copy_(d_i32(p.starts + [200] * (4 - len(p.starts))))
        g.replay()
        want = p.attend()
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(L, want[1])
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for i, x in enumerate((s1, s2) * 3):
        with torch.cuda.stream(x):       # (the outputs are filled there, too)
            outs.append(p.attend(stream=x if i > 1 else None))
    torch.cuda.synchronize()
    for x in outs:
        assert torch.equal(x[0], want[0])
    call = pld.pld_prompt_attn(p.q, p.k, p.v, p.d_starts, o, lse=L, prepare=True)
    o.zero_()
    call()
    assert torch.equal(o, want[0])


def test_attn_refusals():
    p = Prompt([10], 4, 2, 64)
    o = torch.zeros_like(p.q)
    bad = [dict(q=p.q.float()), dict(q=p.q[:, :3]), dict(k=p.k[:5]), dict(v=p.v.transpose(1, 2)), dict(out=o[:, :, ::2]),
           dict(starts=p.d_starts.long()), dict(lse=torch.zeros(10, 2, device=dev())), dict(k=p.k.cpu())]
    for kw in bad:
        args = dict(dict(q=p.q, k=p.k, v=p.v, starts=p.d_starts, out=o), **kw)
        with pytest.raises((TypeError, pld.PLDError)):
            pld.pld_prompt_attn(**args)
    for kw in (dict(scale=-1.0), dict(softcap=NAN), dict(window=-2), dict(out=p.k)):
        with pytest.raises((TypeError, pld.PLDError)):
            pld.pld_prompt_attn(p.q, p.k, p.v, p.d_starts, **{"out": o, **kw})


# ---------------------------------------------------------------------- write
class Write:
    def __init__(self, lens, Hq=4, heads=2, D=64, page=16, dtype=torch.bfloat16, first=None, at=0, pad=0, norm=False, rot=None,
                 axes=0, sections=None, halves=True, seed=0, n_pos=400):
        rng = self.rng = np.random.default_rng(seed)
        self.starts, B = starts_of(lens, at), len(lens)
        N = self.N = max(1, self.starts[-1] + pad)
        self.first = [0] * B if first is None else first
        self.D, self.halves, self.eps = D, halves, 1e-5
        q, k, v = normal(rng, N, (Hq + 2 * heads) * D).split([Hq * D, heads * D, heads * D], -1)
        self.q, self.k, self.v = q.unflatten(-1, (Hq, D)), k.unflatten(-1, (heads, D)), v.unflatten(-1, (heads, D))
        per = max(1, -(-max(f + n for f, n in zip(self.first, lens)) // page))
        self.cache = PagedCache(B, per * page, heads, D, page_size=page, dtype=dtype, num_pages=B * per + 2)
        self.table = rng.permutation(B * per + 2)[:B * per].reshape(B, per).astype(np.int32)
        self.cache.table = d_i32(self.table)
        self.qn, self.kn = (normal(rng, D), normal(rng, D)) if norm else (None, None)
        rot = D if rot is None else rot
        self.rope = self.positions = self.pair_axis = None
        if rot:
            angle = rng.uniform(0, 6.3, (n_pos, rot // 2))
            self.rope = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)).to(dev())
        if axes:
            self.positions = d_i32(rng.integers(0, n_pos, (axes, N)))
            if sections is not None:
                self.pair_axis = d_i32(sections)
        self.d_starts, self.d_first = d_i32(self.starts), d_i32(self.first)
        self.q_out = torch.full_like(self.q.contiguous(), 7.0)
        self.k_out = torch.full_like(self.k.contiguous(), 7.0)

    def write(self, **kw):
        args = dict(q=self.q, k=self.k, v=self.v, starts=self.d_starts, first=self.d_first, q_out=self.q_out, k_out=self.k_out,
                    q_norm=self.qn, k_norm=self.kn, eps=self.eps, rope=self.rope, positions=self.positions, pair_axis=self.pair_axis,
                    rope_pairs=pld.PLD_ROPE_HALVES if self.halves else pld.PLD_ROPE_NEIGHBOURS)
        self.cache.write_packed(**{**args, **kw})

    def expected(self, r, seq):
        """fp64 rows of q and k, None where a position is out of range."""
        pos = self.first[seq] + r - self.starts[seq]
        q, k = (ref.normed(f64(x[r]), None if w is None else f64(w), self.eps) for x, w in ((self.q, self.qn), (self.k, self.kn)))
        if self.rope is not None:
            half = self.rope.shape[1] // 2
            at = [pos] if self.positions is None else self.positions[:, r].tolist()
            axis = [0] * half if self.pair_axis is None else [a if 0 <= a < len(at) else 0 for a in self.pair_axis.tolist()]
            if any(not 0 <= at[a] < self.rope.shape[0] for a in axis):
                return pos, None, None
            q, k = (prompt_ref.turned(x, f64(self.rope), at, axis, self.halves) for x in (q, k))
        return pos, q, k

    def check(self):
        c, q_out, k_out = self.cache, f64(self.q_out), f64(self.k_out)
        q8 = c.k_scale is not None
        kc, vc = f64(c.k), f64(c.v)
        written = np.zeros(kc.shape[:2], bool)
        inside = np.zeros(self.N, bool)
        for b, (a, e) in enumerate(prompt_ref.sequences(self.starts, self.N)):
            inside[a:e] = True
            for r in range(a, e):
                pos, q, k = self.expected(r, b)
                p = pos // c.page_size
                page = self.table[b, p] if 0 <= pos and p < self.table.shape[1] else -1
                if q is None or not 0 <= page < kc.shape[0]:
                    assert np.isnan(q_out[r]).all() and np.isnan(k_out[r]).all(), r
                    continue
                # norm: a sum of D squares, a root and a quotient; rotation: two products and a sum
                tol = lambda x: 2.0 ** -8 * np.abs(x) + (self.D + 16) * U * np.abs(x).max(-1, keepdims=True)
                assert (np.abs(q_out[r] - q) <= tol(q)).all(), r
                assert (np.abs(k_out[r] - k) <= tol(k)).all(), r
                slot = page, pos % c.page_size
                written[slot] = True
                for x, got, scale in ((k, kc, c.k_scale), (f64(self.v[r]), vc, c.v_scale)):
                    if q8:
                        s = f64(scale[slot[0], :, slot[1]])
                        want = np.abs(x).max(-1) / 448
                        assert (np.abs(s - want) <= (self.D + 20) * U * want).all(), r
                        # half a step of e4m3: 2^-4 of a value, and of 2^-6 below that
                        off = np.abs(got[slot] * s[:, None] - x)
                        assert (off <= s[:, None] * (2.0 ** -4 * np.maximum(np.abs(got[slot]), 2.0 ** -6) * 1.01) + tol(x) * 2.0 ** -7).all(), r
                    else:
                        assert (np.abs(got[slot] - x) <= tol(x)).all(), r
        assert (q_out[~inside] == 7).all() and (k_out[~inside] == 7).all()
        assert (kc[~written] == 0).all() and (vc[~written] == 0).all()
        return int(written.sum())


def turns(rot, axes):
    return [t % axes for t in range(rot // 2)]


def sections(rot, axes):
    return [t * axes // (rot // 2) for t in range(rot // 2)]


WRITES = [
    dict(lens=[1]),
    dict(lens=[1, 1, 1], first=[17, 0, 15], axes=3, sections=turns(64, 3)),
    dict(lens=[5, 0, 33, 17], first=[0, 3, 40, 15], at=2, pad=4, axes=3, sections=sections(64, 3), norm=True),
    dict(lens=[20, 30], D=128, Hq=6, heads=3, axes=2, sections=sections(128, 2), halves=False, norm=True),
    dict(lens=[20, 30], D=128, rot=64, axes=4, sections=turns(64, 4), halves=False, dtype=E4M3),
    dict(lens=[40], D=256, axes=3, sections=[0] * 32 + [1] * 48 + [2] * 48, dtype=E4M3, norm=True),
    dict(lens=[40], D=256, rot=0, dtype=E4M3),
    dict(lens=[19, 9], D=128, rot=128, axes=1, page=32, heads=1, Hq=7),
    dict(lens=[19, 9], D=64, rot=24, axes=2, sections=turns(24, 2), norm=True, heads=1, Hq=1),
    dict(lens=[100, 3], D=64, axes=3, sections=[0, 1, 2, 7] * 8, dtype=E4M3, page=64),
]


@pytest.mark.parametrize("case", range(len(WRITES)))
def test_write(case):
    kw = WRITES[case]
    w = Write(seed=case, **kw)
    w.write()
    assert w.check() == sum(kw["lens"])


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("D,halves,rot", [(64, True, 64), (128, False, 64), (128, True, 128), (256, True, 256)])
def test_write_is_the_batched_write(dtype, D, halves, rot):
    """With the cache's positions, or equal ones on all axes: the bits of pld_cache_write."""
    w = Write([7, 4, 30], D=D, dtype=dtype, first=[3, 0, 20], norm=True, rot=rot, halves=halves, seed=2)
    w.write()
    n = 30
    q, k, v = (torch.zeros(3, n, *x.shape[1:], dtype=torch.bfloat16, device=dev()) for x in (w.q, w.k, w.v))
    for b, (a, e) in enumerate(prompt_ref.sequences(w.starts, w.N)):
        for x, y in ((q, w.q), (k, w.k), (v, w.v)):
            x[b, :e - a] = y[a:e]
    other = PagedCache(3, w.cache.table.shape[1] * 16, 2, D, page_size=16, dtype=dtype, num_pages=w.cache.k.shape[0])
    other.table = w.cache.table
    out = torch.zeros_like(q)
    other.write(q, k, v, d_i32([f + 1 for f in w.first]), out, draft_len=d_i32([6, 3, 29]), q_norm=w.qn, k_norm=w.kn, eps=w.eps,
                rope=w.rope, rope_pairs=pld.PLD_ROPE_HALVES if halves else pld.PLD_ROPE_NEIGHBOURS)

    def same():
        assert (bits(other.k) == bits(w.cache.k)).all() and (bits(other.v) == bits(w.cache.v)).all()
        if dtype == E4M3:
            assert (bits(other.k_scale) == bits(w.cache.k_scale)).all() and (bits(other.v_scale) == bits(w.cache.v_scale)).all()
        for b, (a, e) in enumerate(prompt_ref.sequences(w.starts, w.N)):
            assert (bits(out[b, :e - a]) == bits(w.q_out[a:e])).all()
    same()
    at = [f + r - a for f, (a, e) in zip(w.first, prompt_ref.sequences(w.starts, w.N)) for r in range(a, e)]
    w.positions, w.pair_axis = d_i32([at] * 3), d_i32(turns(rot, 3))
    w.cache.k.zero_() if dtype != E4M3 else w.cache.k.view(torch.uint8).zero_()
    w.write()
    same()


def test_write_faults():
    """Bad pages, positions past the table or before the cache, and positions out of the table of angles
    (on an axis that a pair uses, and on one that none does): NaN, and nothing stored."""
    w = Write([30, 20, 5, 4], first=[0, 25, -3, 2000], axes=3, sections=sections(64, 2), norm=True, at=1, pad=1, page=16, seed=4,
              dtype=E4M3)
    assert w.table.shape[1] == 126
    w.table[0, 1], w.table[1, 2] = w.cache.k.shape[0], -1
    w.cache.table = d_i32(w.table)
    w.positions[0, 5], w.positions[1, 7], w.positions[2, 9], w.positions[1, 33] = 400, -1, 100000, 2 ** 31 - 1
    w.write()
    n = w.check()
    # sequence 0 loses page 1 (14 rows) and two positions, 1 page 2 (13 rows) and one position that is not on it or is, 2 three rows
    assert n == (30 - 14 - 2) + (20 - 13 - (1 if 25 + 33 - 31 < 32 else 0)) + (5 - 3) + 4


def test_write_in_place_without_keys_and_far():
    w = Write([50, 20], D=128, first=[0, 5], axes=2, sections=turns(128, 2), norm=True, seed=9)
    w.write()
    q, k = w.q_out.clone(), w.k_out.clone()
    v = Write([50, 20], D=128, first=[0, 5], axes=2, sections=turns(128, 2), norm=True, seed=9)
    v.write(q_out=v.q, k_out=None)
    assert (bits(v.q) == bits(q)).all() and (bits(v.cache.k) == bits(w.cache.k)).all()
    v = Write([50, 20], D=128, first=[0, 5], axes=2, sections=turns(128, 2), norm=True, seed=9)
    v.write(k_out=v.k)
    assert (bits(v.k) == bits(k)).all() and (bits(v.cache.v) == bits(w.cache.v)).all()


def test_write_many_sequences_and_captured():
    """One row of each of 3000 sequences (the single-token form), some empty; captured, with other starts."""
    rng = np.random.default_rng(0)
    lens = (rng.random(3000) < 0.9).astype(int)
    first = [int(x) for x in rng.integers(0, 30, 3000)]
    w = Write(list(lens), first=first, Hq=2, heads=1, axes=3, sections=turns(64, 3), seed=1)
    w.write()
    assert w.check() == lens.sum()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        w.write()
    for _ in range(3):
        lens = (rng.random(3000) < 0.5).astype(int)
        w.starts = starts_of(lens)
        w.d_starts.copy_(d_i32(w.starts))
        w.first = [int(x) for x in rng.integers(0, 30, 3000)]
        w.d_first.copy_(d_i32(w.first))
        for t in (w.q_out, w.k_out):
            t.fill_(7.0)
        for t in (w.cache.k, w.cache.v):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert w.check() == lens.sum()


@pytest.mark.parametrize("kw", [
    # two heads a lane group, and four: head counts that they do not divide, groups that straddle queries, keys and values
    dict(lens=[1500, 1, 0, 1399], Hq=7, heads=1, D=128, axes=3, sections=turns(128, 3), norm=True, at=3, pad=5),
    dict(lens=[700, 560], Hq=6, heads=3, D=256, axes=2, sections=sections(256, 2), halves=False, dtype=E4M3, page=32),
    dict(lens=[2400, 30, 1200], Hq=21, heads=7, D=256, axes=3, sections=turns(256, 3), norm=True, dtype=E4M3, pad=1, page=64),
    dict(lens=[3000, 700], Hq=26, heads=13, D=256, axes=1, rot=128, norm=True, at=1, halves=False, page=128)])
def test_write_several_heads_a_lane_group(kw):
    """Many rows, of which some are not stored: against 64 bits, and by the bits of calls of few rows (a head a lane
    group) into the same cache; in place as well."""
    w = Write(seed=21, n_pos=4000, **kw)
    lanes = w.N * (kw["Hq"] + 2 * kw["heads"]) * w.D // 8
    assert lanes >= 4000000 if kw["Hq"] > 20 else 400000 <= lanes < 4000000        # (where the forms begin)
    # an inner page of the longest sequence, and positions out of the table of angles
    lost = (len(w.table[0]) // 2, w.starts[0] + 5, w.starts[0] + 900 if kw["lens"][0] > 900 else w.starts[1] + 9)
    w.table[0, lost[0]] = -1
    w.cache.table = d_i32(w.table)
    w.positions[0, lost[1]], w.positions[0, lost[2]] = -1, 4000
    q, k = w.q.clone(), w.k.clone()
    w.write()
    assert sum(kw["lens"]) - w.cache.page_size - 2 <= w.check() < sum(kw["lens"])
    outs = lambda: [bits(t) for t in (w.q_out, w.k_out, w.cache.k, w.cache.v, w.cache.k_scale, w.cache.v_scale) if t is not None]
    big = outs()
    for t in (w.cache.k, w.cache.v):
        t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.uint8).zero_()
    w.q_out.fill_(7.0), w.k_out.fill_(7.0)
    step = 390000 * w.N // lanes
    for b, (a, e) in enumerate(prompt_ref.sequences(w.starts, w.N)):
        for x in range(a, e, step):
            y = min(e, x + step)
            w.cache.table = d_i32(w.table[b:b + 1])
            w.write(q=q[x:y], k=k[x:y], v=w.v[x:y], starts=d_i32([0, y - x]), first=d_i32([w.first[b] + x - a]), q_out=w.q_out[x:y],
                    k_out=w.k_out[x:y], positions=w.positions[:, x:y].contiguous())
    for x, y in zip(big, outs()):
        assert np.array_equal(x, y)
    w.cache.table = d_i32(w.table)
    w.write(q_out=w.q, k_out=w.k)
    for x, y, before in ((w.q, big[0], q), (w.k, big[1], k)):
        assert np.array_equal(bits(x)[w.starts[0]:w.starts[-1]], y[w.starts[0]:w.starts[-1]])
        assert torch.equal(x[:w.starts[0]], before[:w.starts[0]]) and torch.equal(x[w.starts[-1]:], before[w.starts[-1]:])
    for x, y in zip(big[2:], outs()[2:]):
        assert np.array_equal(x, y)


def test_write_refusals():
    w = Write([10], axes=2, sections=turns(64, 2))
    for kw in (dict(q=w.q[:, :1]), dict(starts=w.d_starts[:1]), dict(positions=w.positions.long()), dict(positions=w.positions[:, :5]),
               dict(pair_axis=w.pair_axis[:5]), dict(positions=None), dict(k_out=w.k_out[:5]), dict(rope=w.rope[:, :20])):
        with pytest.raises((TypeError, pld.PLDError)):
            w.write(**kw)


# ---------------------------------------------------------------------- pages
class Pages:
    """A pool of `layers` caches beside its model, each with contents of its own everywhere."""

    def __init__(self, seqs, max_pages, num_pages, page=16, layers=2, heads=2, D=64, dtype=torch.bfloat16, layout="slots", seed=0):
        self.rng = np.random.default_rng(seed)
        g = torch.Generator(device=dev()).manual_seed(seed)
        self.model = prompt_ref.Pool(seqs, max_pages, num_pages, page)
        self.k, self.v, self.ks, self.vs = [], [], None, None

        def pages(dtype):
            shape = (num_pages, heads, page, D) if layout == "heads" else (num_pages, page, heads, D)
            x = torch.randint(0, 120, shape, generator=g, device=dev(), dtype=torch.uint8).view(dtype) if dtype == E4M3 else \
                torch.randn(shape, generator=g, device=dev()).to(dtype)
            return x.transpose(1, 2) if layout == "heads" else x
        for _ in range(layers):
            if layout == "pairs":        # keys and values side by side, page by page
                both = torch.randn(num_pages, 2, page, heads, D, generator=g, device=dev()).to(dtype)
                self.k.append(both[:, 0]), self.v.append(both[:, 1])
            else:
                self.k.append(pages(dtype)), self.v.append(pages(dtype))
        if dtype == E4M3:
            self.ks, self.vs = ([torch.rand(num_pages, heads, page, generator=g, device=dev()) for _ in range(layers)] for _ in range(2))
        self.pool = PagePool(self.k, self.v, self.ks, self.vs, table=d_i32(self.model.table), refs=d_i32(self.model.refs))

    def contents(self):
        return [bits(x) for x in self.k + self.v + (self.ks or []) + (self.vs or [])]

    def moved(self, before, copies):
        """`before` with slots of pages copied."""
        n = len(self.k) * 2
        for x, y in enumerate(before):
            for a, b, m in copies:
                if x < n:
                    y[b, :m] = y[a, :m]
                else:
                    y[b, :, :m] = y[a, :, :m]
        return before

    def same(self, contents):
        torch.cuda.synchronize()
        assert np.array_equal(self.pool.table.cpu().numpy(), self.model.table)
        assert np.array_equal(self.pool.refs.cpu().numpy(), self.model.refs)
        for a, b in zip(self.contents(), contents):
            assert np.array_equal(a, b)

    def take(self, seq, need):
        before = self.contents()
        status = torch.full((len(seq),), 9, dtype=torch.int32, device=dev())
        self.pool.take(d_i32(seq), d_i32(need), status)
        want = self.model.take(seq, need)
        assert status.tolist() == want
        self.same(before)
        return want

    def free(self, seq, keep=None):
        before = self.contents()
        self.pool.free(d_i32(seq), None if keep is None else d_i32(keep))
        self.model.free(seq, keep)
        self.same(before)

    def fork(self, src, dst, lens):
        before = self.contents()
        status = torch.full((len(src),), 9, dtype=torch.int32, device=dev())
        self.pool.fork(d_i32(src), d_i32(dst), d_i32(lens), status)
        want, copies = self.model.fork(src, dst, lens)
        assert status.tolist() == want, (status.tolist(), want)
        self.same(self.moved(before, copies))
        return want

    def compact(self, apart=False):
        before = self.contents()
        P = self.model.P
        page_map, used = torch.full((P,), 9, dtype=torch.int32, device=dev()), torch.full((1,), 9, dtype=torch.int32, device=dev())
        if apart:
            t, r = torch.full_like(self.pool.table, 9), torch.full_like(self.pool.refs, 9)
            kept = self.pool.table.clone(), self.pool.refs.clone()
            self.pool.compact(page_map, used, table_out=t, refs_out=r)
            torch.cuda.synchronize()
            assert torch.equal(kept[0], self.pool.table) and torch.equal(kept[1], self.pool.refs)
            self.pool.table.copy_(t), self.pool.refs.copy_(r)
        else:
            self.pool.compact(page_map, used)
        new, n, moves = self.model.compact()
        assert np.array_equal(page_map.cpu().numpy(), new) and used.item() == n
        self.same(self.moved(before, [(a, b, 1 << 20) for a, b in moves]))
        return len(moves)


@pytest.mark.parametrize("kw", [dict(), dict(dtype=E4M3, heads=3), dict(layout="heads", page=32, heads=4), dict(layout="pairs", D=128),
                                dict(layout="heads", dtype=E4M3, layers=3), dict(layers=40, num_pages=40, heads=1), dict(page=128, D=256, layers=1)])
def test_pages_in_random_order(kw):
    """Every call against the pool's model: what is refused, runs short, is named twice."""
    kw = dict(dict(seqs=9, max_pages=6, num_pages=30, seed=len(str(kw))), **kw)
    p = Pages(**kw)
    rng, S, ps = p.rng, kw["seqs"], p.model.ps
    most = kw["max_pages"] * ps
    lens = np.zeros(S, int)
    seen = set()
    for step in range(40):
        n = int(rng.integers(1, 6))
        seq = [int(x) for x in rng.permutation(S)[:n]]
        if step % 7 == 3:
            seq[0] = int(rng.choice([-1, S, seq[-1]]))
        op = ["take", "take", "fork", "free", "keep", "fork", "compact"][step % 7]
        if op == "take":
            need = [int(x) for x in rng.integers(0, most if step > 10 else 2 * ps, n)]
            if step % 5 == 0:
                need[-1] = int(rng.choice([-4, most + 1, 2 ** 31 - 1]))
            seen.update(p.take(seq, need))
        elif op == "fork":
            dst = [int(x) for x in rng.permutation([x for x in range(S) if x not in seq])[:n]]
            seq = seq[:len(dst)]
            if not dst:
                continue
            have = [max([i + 1 for i in range(kw["max_pages"]) if 0 <= s < S and p.model.is_page(p.model.table[s, i])] or [0]) for s in seq]
            t = [int(rng.integers(0, h * ps + 1)) for h in have]
            if step % 3 == 0:
                t[0] = int(rng.choice([-1, most, most + 1]))
            if step % 4 == 0 and len(dst) > 1:
                dst[0] = int(rng.choice([dst[1], seq[1], S]))
            seen.update(p.fork(seq, dst, t))
        elif op == "free":
            p.free(seq + seq[:1])
        elif op == "keep":
            p.free(seq, [int(x) for x in rng.integers(-3, most + 5, n)])
        else:
            p.compact(apart=step % 2 == 0)
    assert {0, -1} <= seen


def test_pages_run_short():
    p = Pages(6, 4, 8)
    assert p.take([0, 1], [48, 33]) == [0, 0]                      # 3 + 3 of 8
    assert p.take([2, 3, 4], [16, 32, 0]) == [0, 2, 0]             # one left of two; that lacks nothing is fine
    assert p.fork([0, 0, 1], [3, 4, 5], [17, 48, 33]) == [0, -2, -2]
    assert p.take([3], [17]) == [0]
    p.free([1, 2])
    assert p.fork([0, 0], [4, 5], [48, 1]) == [0, 0]
    p.free([0, 1, 2, 3, 4, 5])
    assert (p.model.refs == 0).all()
    assert p.compact() == 0


def test_pages_of_a_large_pool():
    """Several blocks of references, and more table entries than one block goes through."""
    p = Pages(300, 200, 40000, layers=1, heads=1, seed=3)
    rng = p.rng
    seqs = [int(x) for x in rng.permutation(300)]
    assert p.take(seqs, [int(x) for x in rng.integers(0, 200 * 16, 300)]).count(0) == 300
    p.free(seqs[:120], [int(x) for x in rng.integers(0, 1500, 120)])
    src, dst = seqs[200:290], seqs[:90]
    assert p.fork(src, dst, [int(min(40, 16 * (p.model.table[s] >= 0).sum())) for s in src]).count(0) == 90
    assert p.take(seqs[:200], [3000] * 200)[-1] > 0                 # not enough for all
    p.free(seqs[60:180])
    assert p.compact(apart=True) > 1000
    assert p.take([5], [3200]) == [0]


@pytest.mark.parametrize("n", [1, 3, 20])
def test_pages_of_long_sequences(n):
    """More entries a sequence than a wave takes at a time, by one block's waves and by launches of their own."""
    p = Pages(3 * n, 1500, 2200 * n, layers=1, heads=1, seed=n)
    rng, own, new = p.rng, list(range(n)), list(range(n, 2 * n))
    assert p.take(own, [int(x) for x in rng.integers(513 * 16, 1100 * 16, n)]) == [0] * n
    held = [int((p.model.table[s] >= 0).sum()) for s in own]
    lens = [int(rng.integers((h - 20) * 16, h * 16)) for h in held]
    assert p.fork(own, new, lens) == [0] * n
    assert p.take(new, [x + 700 for x in lens]) == [0] * n
    p.free(own, [int(rng.integers(0, 600 * 16)) for _ in own])
    p.model.table[new[0], 5:700:3] = -1                             # entries that name no page, some out of range
    p.model.table[new[0], 6:700:9] = 1 << 30
    p.pool.table.copy_(d_i32(p.model.table))
    used = np.unique(p.model.table[(p.model.table >= 0) & (p.model.table < p.model.P)], return_counts=True)
    p.model.refs[:] = 0
    p.model.refs[used[0]] = used[1]
    p.pool.refs.copy_(d_i32(p.model.refs))
    assert p.fork(new, list(range(2 * n, 3 * n)), lens) == [0] * n
    p.take(list(range(2 * n, 3 * n)), [1500 * 16] * n)              # whole tables, as far as there are pages
    p.take(new, [x + 3000 for x in lens])
    p.compact(apart=True)
    p.free(list(range(3 * n)), [600 * 16] * 3 * n)


def test_pages_held_by_the_caller():
    """A page with a reference of the caller's own stays in use, and moves."""
    p = Pages(2, 3, 9)
    for x in (4, 8):
        p.model.refs[x] = 1
    p.pool.refs.copy_(d_i32(p.model.refs))
    p.take([0], [48])
    p.free([0])
    assert p.compact() == 2


def test_fork_integers_alone_and_captured():
    p = Pages(4, 4, 16, layers=2)
    p.take([0], [60])
    status, src, lens = torch.zeros(2, dtype=torch.int32, device=dev()), d_i32([0, 0]), d_i32([50, 20])
    seq, need, taken = d_i32([1, 2]), d_i32([64, 40]), torch.zeros(2, dtype=torch.int32, device=dev())
    pool = p.pool
    pool.reserve(2)
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        pool.free(seq)
        pool.fork(src, seq, lens, status)
        pool.take(seq, need, taken)
    for t in ([50, 20], [1, 60], [33, 32]):
        lens.copy_(d_i32(t))
        before = p.contents()
        g.replay()
        torch.cuda.synchronize()
        p.model.free([1, 2])
        want, copies = p.model.fork([0, 0], [1, 2], t)
        assert p.model.take([1, 2], [64, 40]) == taken.tolist() and want == status.tolist() == [0, 0]
        p.same(p.moved(before, copies))
    none = pld.PageLayers([], [])
    before = p.contents()
    pld.pld_pages_fork(pool.pages, none, src, seq, lens, status, pool.workspace)
    p.model.fork([0, 0], [1, 2], [33, 32])
    p.same(before)


@pytest.mark.parametrize("a,b", [("slots", "heads"), ("heads", "slots"), ("heads", "heads"), ("slots", "slots"), ("pairs", "slots")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
def test_copy_between_layouts(a, b, dtype):
    if dtype == E4M3 and "pairs" in (a, b):
        pytest.skip("a layout of bfloat16 alone here")
    kw = dict(seqs=1, max_pages=1, page=32, heads=3, D=128, dtype=dtype)
    x, y = Pages(num_pages=9, layout=a, seed=1, **kw), Pages(num_pages=12, layout=b, seed=2, **kw)
    src, dst, slots = [0, 8, 3, 9, 5, 2, 1], [11, 0, 4, 5, -1, 6, 7], [32, 1, 17, 32, 32, 0, -5]
    for s in (slots, None):
        want = y.contents()
        for f, t in zip(x.contents(), want):
            for i, j, m in zip(src, dst, s or [32] * 7):
                if 0 <= i < 9 and 0 <= j < 12:
                    m = m if 0 <= m <= 32 else 32
                    t[j, ..., :m] = f[i, ..., :m] if t.ndim == 3 else t[j, ..., :m]
                    if t.ndim == 4:
                        t[j, :m] = f[i, :m]
        y.pool.copy_from(x.pool, d_i32(src), d_i32(dst), None if s is None else d_i32(s))
        torch.cuda.synchronize()
        for got, t in zip(y.contents(), want):
            assert np.array_equal(got, t)


def _layers(layout, dtype, P, page, heads, D, seed):
    """Two layers' keys, values and scales in one of several layouts."""
    g = torch.Generator(device=dev()).manual_seed(seed)

    def rows(*shape):
        return torch.randint(0, 120, shape, generator=g, device=dev(), dtype=torch.uint8).view(E4M3) if dtype == E4M3 else \
            torch.randn(shape, generator=g, device=dev()).to(dtype)

    def pair():
        if layout == "heads":                                  # slot by slot within a head
            return [rows(P, heads, page, D).transpose(1, 2) for _ in range(2)]
        if layout == "pairs":                                  # keys and values side by side, page by page
            both = rows(P, 2, page, heads, D)
            return [both[:, 0], both[:, 1]]
        if layout == "slots together":                         # keys and values side by side, slot by slot
            both = rows(P, page, 2, heads, D)
            return [both[:, :, 0], both[:, :, 1]]
        return [rows(P, page, heads, D) for _ in range(2)]
    pairs = [pair() for _ in range(2)]
    k, v = [x[0] for x in pairs], [x[1] for x in pairs]
    scales = [[torch.rand(P, heads, page, generator=g, device=dev()) for _ in range(2)] for _ in range(2)] if dtype == E4M3 else (None, None)
    return k, v, *scales


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("a,b", [("slots", "heads"), ("heads", "heads"), ("heads", "slots"), ("pairs", "slots together"),
                                 ("slots together", "heads"), ("slots", "pairs")])
def test_copy_of_large_pages(a, b, dtype):
    """Pages of several parts of 32 KB, whole and partly, between layouts that are no single run of bytes."""
    page, heads, D = 256, 5, 128
    x, y = _layers(a, dtype, 7, page, heads, D, 1), _layers(b, dtype, 6, page, heads, D, 2)
    src, dst, slots = [6, 0, 3, 5, 2], [0, 5, 2, 4, 1], [256, 255, 65, 1, 0]
    for s in (slots, None):
        want = [[bits(t) for t in list_] for list_ in y if list_]
        for from_, to in zip([list_ for list_ in x if list_], want):
            for f, t in zip((bits(f) for f in from_), to):
                for i, j, m in zip(src, dst, s or [page] * 5):
                    if t.ndim == 4:
                        t[j, :m] = f[i, :m]
                    else:
                        t[j, :, :m] = f[i, :, :m]
        PagePool(*y).copy_from(PagePool(*x), d_i32(src), d_i32(dst), None if s is None else d_i32(s))
        torch.cuda.synchronize()
        for got, to in zip([list_ for list_ in y if list_], want):
            for g, t in zip(got, to):
                assert np.array_equal(bits(g), t)


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("layout", ["heads", "pairs", "slots together"])
def test_fork_and_compact_large_pages(layout, dtype):
    """The tail of a fork and a compaction's moves, of several parts of 32 KB a page."""
    page, heads, D = 256, 5, 128
    x = _layers(layout, dtype, 8, page, heads, D, 3)
    contents = lambda: [bits(t) for list_ in x if list_ for t in list_]
    pool = PagePool(*x, table=d_i32([[6, 7, -1], [-1] * 3, [1, -1, -1]]), refs=d_i32([0, 1, 0, 0, 0, 0, 1, 1]))
    status = d_i32([9])
    for call, moves in ((lambda: pool.fork(d_i32([0]), d_i32([1]), d_i32([page + 77]), status), [(7, 0, 77)]),
                        (lambda: pool.compact(d_i32([0] * 8), d_i32([0])), [(6, 2, page), (7, 3, page)])):
        want = contents()
        for t in want:
            for i, j, m in moves:
                if t.ndim == 4:
                    t[j, :m] = t[i, :m]
                else:
                    t[j, :, :m] = t[i, :, :m]
        call()
        torch.cuda.synchronize()
        for g, t in zip(contents(), want):
            assert np.array_equal(g, t)
    assert status.item() == 0 and pool.table.tolist() == [[2, 3, -1], [2, 0, -1], [1, -1, -1]]
    assert pool.refs.tolist() == [1, 1, 2, 1, 0, 0, 0, 0]


def test_copy_far_pages():
    """Offsets past 2^31 bytes on both sides."""
    P, page = 700, 4096
    mk = lambda: torch.zeros(P, page, 8, 128, dtype=torch.bfloat16, device=dev())      # 5.9 GB
    k, v = mk(), mk()
    pool = PagePool([k], [v])
    k[650] = torch.randn(page, 8, 128, device=dev()).to(torch.bfloat16)
    v[3, :100] = 1.5
    pool.copy_from(pool, d_i32([650, 3]), d_i32([2, 699]), d_i32([4000, 4096]))
    torch.cuda.synchronize()
    assert torch.equal(k[2, :4000], k[650, :4000]) and (k[2, 4000:] == 0).all()
    assert torch.equal(v[699], v[3]) and (v[2] == 0).all()


def test_compacting_and_copying_captured():
    """The same graph over other contents of the pool, eager calls between the replays."""
    p = Pages(5, 4, 24, layers=2, seed=2)
    page_map, used = torch.zeros(24, dtype=torch.int32, device=dev()), torch.zeros(1, dtype=torch.int32, device=dev())
    p.pool.reserve(5)
    src, dst, slots = d_i32([0, 1]), d_i32([22, 23]), d_i32([16, 3])
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        p.pool.compact(page_map, used)
        p.pool.copy_from(p.pool, src, dst, slots)
    for ended in ([0], [1, 3], [], [2, 4], [0, 1, 2, 3, 4]):
        p.take([0, 1, 2, 3, 4], [60, 17, 33, 1, 64])
        if ended:                      # (a call names one at least)
            p.free(ended)
        before = p.contents()
        g.replay()
        new, n, moves = p.model.compact()
        p.moved(before, [(a, b, 1 << 20) for a, b in moves])
        p.same(p.moved(before, [(0, 22, 16), (1, 23, 3)]))
        assert np.array_equal(page_map.cpu().numpy(), new) and used.item() == n


def test_prepared_page_calls():
    """Calls marshalled once, issued again and again."""
    p = Pages(4, 4, 20)
    pool, one = p.pool, d_i32([0])
    seq, lens, status = d_i32([1, 2]), d_i32([40, 33]), torch.zeros(2, dtype=torch.int32, device=dev())
    page_map, used = torch.zeros(20, dtype=torch.int32, device=dev()), torch.zeros(1, dtype=torch.int32, device=dev())
    p.take([0], [60])
    src, need, to, keep, taken = d_i32([0, 0]), d_i32([60]), d_i32([19]), d_i32([40]), d_i32([9])
    calls = [pool.fork(src, seq, lens, status, prepare=True), pool.free(one, keep, prepare=True),
             pool.compact(page_map, used, prepare=True), pool.take(one, need, taken, prepare=True)]
    copy = pool.copy_from(pool, one, to, prepare=True)
    pool.reserve(50)                       # (the calls keep the workspace that they were made with)
    for _ in range(3):
        before = p.contents()
        calls[0]()
        want, copies = p.model.fork([0, 0], [1, 2], [40, 33])
        assert status.tolist() == want == [0, 0]
        p.same(p.moved(before, copies))
        calls[1](), p.model.free([0], [40])
        calls[2]()
        new, n, moves = p.model.compact()
        p.same(p.contents())               # (contents in test_pages_in_random_order)
        assert np.array_equal(page_map.cpu().numpy(), new) and used.item() == n
        calls[3]()
        assert p.model.take([0], [60]) == taken.tolist() == [0]
        before = p.contents()
        copy()
        p.same(p.moved(before, [(0, 19, 16)]))


def test_pool_refusals():
    p = Pages(3, 4, 8)
    i = d_i32([0])
    for call in (lambda: p.pool.take(i, i.long(), i), lambda: p.pool.take(i, d_i32([1, 2]), i), lambda: p.pool.free(i.cpu()),
                 lambda: p.pool.fork(i, i, i, d_i32([0, 0])), lambda: p.pool.compact(i, i),
                 lambda: p.pool.compact(d_i32([0] * 8), i, table_out=p.pool.table[:2]),
                 lambda: p.pool.copy_from(Pages(3, 4, 8, layers=1).pool, i, i), lambda: p.pool.copy_from(Pages(3, 4, 8, heads=1).pool, i, i),
                 lambda: pld.PageLayers([p.k[0], p.k[1][:4]], p.v), lambda: pld.pld_pages_take(p.pool.pages, i, i, i, i),
                 lambda: pld.PageTable(p.pool.table, p.pool.refs.float(), 16), lambda: pld.PageTable(p.pool.table[0], p.pool.refs, 16)):
        with pytest.raises((TypeError, pld.PLDError)):
            call()


def test_compact_refuses_rows_that_overlap():
    p = Pages(3, 4, 8)
    page_map, used = d_i32([9] * 8), d_i32([9])
    for t in (d_i32([0] * 4).expand(3, 4), d_i32([0] * 12).as_strided((3, 4), (3, 1))):
        with pytest.raises(pld.PLDError):
            p.pool.compact(page_map, used, table_out=t)
        with pytest.raises(pld.PLDError):
            PagePool(p.k, p.v, table=t, refs=p.pool.refs).compact(page_map, used)
    assert (page_map == 9).all() and used.item() == 9


def test_a_refused_page_call_leaves_the_pool_usable():
    """More entries than a call takes are refused; the calls that follow are as without it."""
    p = Pages(6, 4, 20)
    many = d_i32([0] * (pld.PLD_MAX_PAGE_ENTRIES + 1))
    for call in (lambda: p.pool.take(many, many, many), lambda: p.pool.fork(many, many, many, many), lambda: p.pool.free(many)):
        with pytest.raises(pld.PLDError):
            call()
    assert p.take([0, 1], [40, 17]) == [0, 0]
    with pytest.raises(pld.PLDError):
        p.pool.take(many, many, many)
    assert p.fork([0, 1], [2, 3], [40, 9]) == [0, 0]
    p.free([0])
    assert p.compact() > 0


@pytest.mark.parametrize("other", [dict(num_pages=9), dict(heads=1), dict(dtype=E4M3), dict(page_size=32)])
def test_a_refused_pool_leaves_its_caches_as_they_were(other):
    make = lambda **kw: PagedCache(**{**dict(B=2, max_len=40, heads=2, head_dim=64, page_size=16), **kw})
    caches = [make(), make(**other)]
    tables = [c.table for c in caches]
    with pytest.raises(TypeError):
        PagePool.of_caches(caches, seqs=3)
    assert all(c.table is t for c, t in zip(caches, tables))
    pool = PagePool.of_caches(caches[:1], seqs=3)
    assert caches[0].table is pool.table and pool.table.shape == (3, 3)


# ------------------------------------------------------------- a run of them
@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
def test_prompts_forks_and_verification(dtype):
    """Prompts packed into a pool's pages and attended to, the cache's attention over the same rows; each
    prompt goes on in two sequences that share its pages, whose verification passes write and attend as
    a sequence of its own does, before and after the pool is compacted."""
    rng = np.random.default_rng(0)
    lens, Hq, heads, D, page = [70, 33, 16, 128], 8, 2, 64, 16
    B, n = len(lens), 5
    per = -(-(max(lens) + 20) // page)
    cache = PagedCache(B, per * page, heads, D, page_size=page, dtype=dtype, num_pages=4 * B * per)
    pool = PagePool.of_caches([cache], seqs=3 * B + B, max_len=per * page)
    status = torch.full((3 * B + B,), 9, dtype=torch.int32, device=dev())
    order = d_i32(list(range(B)))

    w = Write(lens, Hq=Hq, heads=heads, D=D, axes=3, sections=turns(64, 3), norm=True, seed=5)
    w.cache = cache
    pool.take(order, d_i32(lens), status[:B])
    assert (status[:B] == 0).all()
    whole = pool.table
    cache.table = whole[:B]
    w.write()
    out, lse = torch.zeros_like(w.q_out), torch.zeros(w.N, Hq, device=dev())
    pld.pld_prompt_attn(w.q_out, w.k_out, w.v, w.d_starts, out, lse=lse)
    # (the cache's attention takes a prompt as rows from position 0 on)
    m = max(lens)
    q = torch.zeros(B, m, Hq, D, dtype=torch.bfloat16, device=dev())
    for b, (a, e) in enumerate(prompt_ref.sequences(w.starts, w.N)):
        q[b, :e - a] = w.q_out[a:e]
    o2, l2 = torch.zeros_like(q), torch.zeros(B, m, Hq, device=dev())
    cache.attend(q, d_i32([1] * B), o2, draft_len=d_i32([x - 1 for x in lens]), lse=l2)
    for b, (a, e) in enumerate(prompt_ref.sequences(w.starts, w.N)):
        if dtype != torch.bfloat16:
            continue                 # (its keys and values are rounded, the prompt's are not)
        # both are within out_bound and lse_bound of the same 64-bit values; sums of weights times |v| are at most the largest |v|
        x, y, z = f64(w.q_out[a:e]), f64(w.k_out[a:e]), f64(w.v[a:e])
        size = max((np.abs(x[:, h]) @ np.abs(y[:, h // 4]).T).max() for h in range(Hq)) * D ** -0.5
        tol, top = (D + 8) * U * size, np.abs(z).max()
        assert np.abs(f64(out[a:e]) - f64(o2[b, :e - a])).max() <= 2 * ref.out_bound(top, top, tol)
        assert (lse[a:e] - l2[b, :e - a]).abs().max() <= 2 * ref.lse_bound(tol, float(lse[a:e].abs().max()), e - a)
    # two sequences go on from each prompt, and a third that is a copy of its own, page by page
    src = order.repeat(2)
    dst = d_i32(list(range(B, 3 * B)))
    pool.fork(src, dst, d_i32(lens * 2), status[:2 * B])
    own = d_i32(list(range(3 * B, 4 * B)))
    pool.take(own, d_i32(lens), status[2 * B:3 * B])
    assert (status[:3 * B] == 0).all()
    pairs = [(int(whole[b, p]), int(whole[3 * B + b, p])) for b in range(B) for p in range(-(-lens[b] // page))]
    pool.copy_from(pool, d_i32([a for a, _ in pairs]), d_i32([b for _, b in pairs]))
    go = torch.cat([dst, own])
    pool.take(go, d_i32([x + n for x in lens] * 3), status[:3 * B])
    assert (status[:3 * B] == 0).all()
    assert (pool.refs > 1).sum() == sum((x - 1) // page for x in lens)

    q, k, v = normal(rng, B, n, Hq, D), normal(rng, B, n, heads, D), normal(rng, B, n, heads, D)
    q2, k2, v2 = (normal(rng, *x.shape) for x in (q, k, v))
    rows = d_i32(lens)

    def verify(first, q, k, v):
        cache.table = pool.table[first:first + B]
        o, out = torch.zeros_like(q), torch.zeros_like(q)
        cache.write(q, k, v, rows, out)
        cache.attend(out, rows, o)
        return o

    a, b = verify(B, q, k, v), verify(2 * B, q2, k2, v2)
    c, d = verify(3 * B, q, k, v), verify(B, q, k, v)
    assert torch.equal(a, c) and torch.equal(a, d) and not torch.equal(a, b)
    # single tokens by the packed write go where the batched write puts them
    one = torch.zeros(B, Hq, D, dtype=torch.bfloat16, device=dev())
    before = bits(cache.k)
    cache.write_packed(q[:, 0], k[:, 0], v[:, 0], d_i32(range(B + 1)), d_i32([x - 1 for x in lens]), one)
    assert (bits(cache.k) == before).all() and torch.equal(one, q[:, 0])
    # the prompts' own sequences end, and the pool is compacted: nobody notices
    pool.free(order)
    page_map = torch.zeros(cache.k.shape[0], dtype=torch.int32, device=dev())
    used = torch.zeros(1, dtype=torch.int32, device=dev())
    pool.free(own)
    pool.compact(page_map, used)
    assert int(pool.table.max()) < used.item() == int((pool.refs > 0).sum())
    cache.table = pool.table[B:2 * B]
    o = torch.zeros_like(a)
    cache.attend(q, rows, o)
    assert torch.equal(o, a)
    cache.table = pool.table[2 * B:3 * B]
    cache.attend(q2, rows, o)
    assert torch.equal(o, b)
    pool.free(dst)
    assert (pool.refs == 0).all() and (pool.table == -1).all()
