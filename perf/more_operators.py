"""A prompt's pass and the pages it fills: the operators' cases, their plain forms and their values in 64 bits.

Prompts of different lengths are read together, their rows packed: row r belongs to sequence b where starts[b] <= r <
starts[b+1]; rows behind the last sequence stay as they are.  Keys and values join a layer's paged cache, the rows attend
to each other, and what one prompt has filled is shared by the sequences that go on from it.

  write    x / sqrt(mean(x^2) + eps) * w per head, pair t of the first `rot` elements turned by the angle of the row's
           position on axis pair_axis[t]; queries (and keys, for the attention) back to the program, keys and values to
           the slots of positions first[b], first[b] + 1, ... (e4m3: one scale a row and head)
  attn     softmax over keys r - window < j <= r of the row's own sequence, of cap * tanh(q.k * scale / cap), times v;
           with its log sum
  fork     a scheduler's step: sequences that ended give their pages back (refs counts the table entries that name a
           page), others go on in their place from a prompt's first lens tokens - whole pages before the one of the last
           token are shared, that one's slots are copied in every layer - and get pages for their next tokens, lowest first
  compact  pages in use move to the lowest indices, order kept where they have to move; the table follows
  copy     pages between two caches, the first slots[i] slots of each, in every layer
"""
import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0


# ------------------------------------------------------------------ cases
def _case(name=None, *, op, B, T, ragged=0.0, pad=0, Hq=0, Hkv=0, D=0, softcap=0.0, window=0, page=0, cache="", past=0, rot=0,
          pairs="halves", axes=1, turns=False, norm=False, layers=1, count=0, spare=0, ahead=0):
    """B, T: sequences and the longest one's tokens (ragged: the shortest has (1 - ragged) T); pad: rows behind the last
    sequence; past: tokens of the longest sequence that the cache holds already; turns: the axes take turns from pair to
    pair, else each has a section; layers: caches of the pool; count: forks, or pages to copy; spare: free pages among the
    used ones, in percent; ahead: tokens that the forked sequences get pages for."""
    c = dict(op=op, B=B, T=T, ragged=ragged, pad=pad, Hq=Hq, Hkv=Hkv, D=D, softcap=softcap, window=window, page=page, cache=cache,
             past=past, rot=rot, pairs=pairs, axes=axes, turns=turns, norm=norm, layers=layers, count=count, spare=spare, ahead=ahead)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # one user's short question: launch and latency
        _case("attn_b1_t71", op="attn", B=1, T=71, Hq=32, Hkv=8, D=128),
        # a serving batch of prompts of many lengths, packed into a buffer that is a little larger
        _case("attn_b8_t4096_ragged", op="attn", B=8, T=4096, ragged=0.9, pad=37, Hq=32, Hkv=8, D=128),
        # narrow heads, capped scores in a window, odd lengths
        _case("attn_b12_t3333_window", op="attn", B=12, T=3333, ragged=0.7, Hq=24, Hkv=4, D=64, softcap=30.0, window=1000),
        # one long document beside short ones
        _case("attn_b3_t32768", op="attn", B=3, T=32768, ragged=0.99, Hq=32, Hkv=8, D=128),
        # one user's next token after images in its prompt
        _case("write_b1_token", op="write", B=1, T=1, Hq=32, Hkv=8, D=128, page=16, cache="bf16", past=1024, rot=128, axes=3, norm=True),
        # prompts with images into a quantised cache, axes in turns
        _case("write_b6_t4096_e4m3", op="write", B=6, T=4096, ragged=0.6, pad=19, Hq=32, Hkv=8, D=128, page=64, cache="e4m3", rot=128, axes=3,
              turns=True, norm=True),
        # a second sequence from one short prompt, one layer
        _case("fork_b1", op="fork", B=1, T=1024, Hkv=8, D=128, page=16, cache="bf16", count=1, ahead=17),
        # a step of a large batch: eight prompts' sequences replaced, sixteen layers
        _case("fork_b56_l16", op="fork", B=8, T=4096, ragged=0.5, Hkv=8, D=128, page=64, cache="bf16", layers=16, count=56, ahead=100),
        # a small pool after one sequence ended
        _case("compact_b2", op="compact", B=2, T=500, ragged=0.5, Hkv=8, D=128, page=16, cache="bf16", spare=40),
        # a large pool, half of it free, quantised
        _case("compact_b32_l8_e4m3", op="compact", B=32, T=8192, ragged=0.8, Hkv=8, D=128, page=64, cache="e4m3", layers=8, spare=50),
        # one short prompt's pages into another cache
        _case("copy_b1", op="copy", B=1, T=300, Hkv=8, D=128, page=16, cache="bf16", count=19),
        # a long document's pages out of every layer, the last one not full
        _case("copy_b1_t65000_l16", op="copy", B=1, T=65000, Hkv=8, D=128, page=32, cache="bf16", layers=16, count=2032),
    ]


def _spread(rng, lo, hi):
    """A whole number, its logarithm uniform over [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["attn", "attn", "attn", "write", "write", "fork", "compact", "copy"])
        heads, group, D = rng.choice([1, 2, 4, 8, 8, 16, 32]), rng.choice([1, 2, 4, 5, 6, 7, 8, 12, 16]), rng.choice([64, 128, 128, 256])
        c = dict(op=op, B=_spread(rng, 1, 64), ragged=rng.choice([0.0, round(rng.uniform(0.1, 0.99), 2)]), Hkv=heads, D=D)
        if op in ("attn", "write"):
            c.update(Hq=heads * group, pad=rng.choice([0, 0, rng.randint(1, 300)]))
        if op != "attn":
            c.update(page=rng.choice([16, 32, 64, 128]), cache=rng.choice(["bf16", "e4m3"]))
        if op == "attn":
            cap, window = rng.choice([(0.0, 0), (0.0, 0), (30.0, 0), (0.0, _spread(rng, 1, 8000)), (50.0, _spread(rng, 16, 8000))])
            c.update(T=_spread(rng, 1, 32768), softcap=cap, window=window)
        elif op == "write":
            c.update(T=rng.choice([1, _spread(rng, 1, 17), _spread(rng, 1, 16000)]), past=rng.choice([0, _spread(rng, 1, 2000)]),
                     rot=rng.choice([D, D // 2, 0]), pairs=rng.choice(["halves", "neighbours"]), axes=rng.choice([1, 2, 3, 3, 4]),
                     turns=rng.random() < 0.5, norm=rng.random() < 0.5)
        else:
            c.update(T=_spread(rng, 1, 65536), layers=_spread(rng, 1, 32), spare=rng.choice([10, 40, 50, 70]), count=0)
            if op == "fork":
                c.update(count=_spread(rng, 1, 64), ahead=_spread(rng, 1, 300))
            if op == "copy":
                c.update(B=1, ragged=0.0, count=-(-c["T"] // c["page"]))
        c = _case(**c)
        w, most = work(c), _most[op]
        if c["Hq"] > 128 or w["bytes"] > most["bytes"] or w["flops"] > most["flops"] or _held(c) > 6.4e9 or _rows(c) > 100000:
            continue
        return c


# ------------------------------------------------------------------ what a pass cannot do without
def _lens(c):
    B, T = c["B"], c["T"]
    return [T - int(c["ragged"] * (T - 1) * b / max(1, B - 1)) for b in range(B)]


def _rows(c):
    """Rows of the packed buffers."""
    return sum(_lens(c)) + c["pad"] if c["Hq"] else 0


def _table(c):
    """Table entries of a sequence."""
    return -(-(c["past"] + c["T"] + c["ahead"]) // c["page"])


def _pool(c):
    """Pages of the pool."""
    used = sum(-(-(c["past"] + t) // c["page"]) for t in _lens(c))
    if c["op"] == "fork":
        return used + c["count"] * (3 + -(-c["ahead"] // c["page"])) + 5
    if c["op"] == "compact":
        return -(-used * 100 // (100 - c["spare"])) + 3
    return c["B"] * _table(c) + 2


def _row(c):
    """Bytes of one head's key or value of one token in the cache."""
    return 2 * c["D"] if c["cache"] == "bf16" else c["D"] + 4


def _held(c):
    """Bytes of the caches, or of the packed rows."""
    if not c["page"]:
        return 2 * _rows(c) * c["D"] * (2 * c["Hq"] + 2 * c["Hkv"])
    return 2 * _pool(c) * c["page"] * c["Hkv"] * _row(c) * c["layers"] * (2 if c["op"] == "copy" else 1)


def _moved(c):
    """Pages at or above the number of used ones, which have to move: the pages that are free are spread evenly."""
    used = sum(-(-t // c["page"]) for t in _lens(c))
    return used * (_pool(c) - used) // _pool(c)


def work(case):
    c = case
    lens, D, Hq, Hkv = _lens(c), c["D"], c["Hq"], c["Hkv"]
    rows = sum(lens)
    slot = 2 * Hkv * _row(c) * c["layers"] if c["cache"] else 0       # a token's keys and values
    if c["op"] == "attn":
        w = c["window"]
        seen = sum(t * (t + 1) // 2 if not w or t <= w else w * (w + 1) // 2 + (t - w) * w for t in lens)
        return {"bytes": rows * (4 * D * Hq + 4 * D * Hkv + 4 * Hq), "flops": 4 * D * Hq * seen}
    if c["op"] == "write":
        table = min(rows, c["T"]) * c["rot"] * 4 + rows * 4 * c["axes"]
        return {"bytes": rows * (4 * D * Hq + 6 * D * Hkv + 2 * _row(c) * Hkv) + table, "flops": rows * D * (Hq + 2 * Hkv) * 8}
    if c["op"] == "fork":
        tails = sum((lens[i % c["B"]] - 1) % c["page"] + 1 for i in range(c["count"]))
        return {"bytes": 2 * tails * slot + (c["count"] * 3 * _table(c) + _pool(c)) * 4, "flops": 0}
    if c["op"] == "compact":
        return {"bytes": 2 * _moved(c) * c["page"] * slot + (2 * c["B"] * _table(c) + 3 * _pool(c)) * 4, "flops": 0}
    return {"bytes": 2 * c["T"] * slot + c["count"] * 12, "flops": 0}


_most = {}
for _c in listed():
    _w = work(_c)
    _most[_c["op"]] = {k: max(v, _most.get(_c["op"], _w)[k]) for k, v in _w.items()}


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    i32 = dict(dtype=torch.int32, device="cuda")
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)
    B, Hq, Hkv, D, page = c["B"], c["Hq"], c["Hkv"], c["D"], c["page"]
    mix = torch.randperm(B, generator=g, device="cuda")                            # which sequence has which length
    lens = torch.tensor(_lens(c), **i32)[mix]
    s = dict(case=c, lens=lens)
    if Hq:
        # one projection's output: q, k and v of a row side by side
        N, rows = _rows(c), sum(_lens(c))
        s["starts"] = torch.cat([torch.zeros(1, **i32), lens.cumsum(0).to(torch.int32)])
        s["rows"] = rows
        q, k, v = normal(N, (Hq + 2 * Hkv) * D).split([Hq * D, Hkv * D, Hkv * D], -1)
        if c["op"] == "attn":
            q.mul_(2)
        s["q"], s["k"], s["v"] = q.unflatten(-1, (Hq, D)), k.unflatten(-1, (Hkv, D)), v.unflatten(-1, (Hkv, D))
        s["out"] = torch.zeros(N, Hq, D, dtype=torch.bfloat16, device="cuda")
    if c["op"] == "attn":
        s["lse"] = torch.zeros(N, Hq, device="cuda")
        return s
    P, L, per = _pool(c), c["layers"], _table(c)
    if c["op"] == "write":
        s["table"] = torch.randperm(P, generator=g, device="cuda")[:B * per].to(torch.int32).view(B, per)
        _caches(s, c, normal, "", 1, P)
        s["first"] = torch.tensor([c["past"] - c["past"] * b // max(1, B) for b in range(B)], **i32)[mix]
        s["k_out"] = torch.zeros(N, Hkv, D, dtype=torch.bfloat16, device="cuda")
        s["q_norm"] = s["k_norm"] = s["rope"] = s["positions"] = s["pair_axis"] = None
        if c["norm"]:
            s["q_norm"], s["k_norm"] = normal(D).mul_(0.1).add_(1), normal(D).mul_(0.1).add_(1)
        if c["rot"]:
            # text and images of 16 x 16 patches in turns: 256 positions on all axes, then one in time by 16 by 16 in the others
            seq = torch.repeat_interleave(torch.arange(B, device="cuda"), lens.long(), output_size=rows)
            r = torch.arange(rows, device="cuda") - s["starts"].long()[seq]
            part, at = r // 256, r % 256
            base, image = s["first"].long()[seq] + part // 2 * 272 + part % 2 * 256, part % 2 == 1
            axis = [torch.where(image, x, at) + base for x in (0 * at, at // 16, at % 16, 0 * at)]
            s["positions"] = torch.zeros(c["axes"], N, **i32)
            s["positions"][:, :rows] = torch.stack(axis[:c["axes"]]).to(torch.int32)
            pair = torch.arange(c["rot"] // 2, device="cuda")
            s["pair_axis"] = (pair % c["axes"] if c["turns"] else pair * c["axes"] // (c["rot"] // 2)).to(torch.int32)
            freq = 500000.0 ** (-2 * pair.to(torch.float64) / c["rot"])
            angle = torch.arange(c["past"] + c["T"], dtype=torch.float64, device="cuda")[:, None] * freq
            s["rope"] = torch.cat([angle.cos(), angle.sin()], -1).float()
        return s
    _caches(s, c, normal, "", L, P)
    held = -(-lens // page)                                                        # pages of each prompt
    if c["op"] == "copy":
        _caches(s, c, normal, "to_", L, P)
        n = c["count"]
        s["src"], s["dst"] = (torch.randperm(P, generator=g, device="cuda")[:n].to(torch.int32) for _ in range(2))
        s["slots"] = (c["T"] - page * torch.arange(n, **i32)).clamp(max=page)
        return s
    # the prompts' pages lie anywhere in the pool, where its last users left room
    S = B + c["count"]
    s["table"] = torch.full((S, per), -1, **i32)
    mine = torch.arange(per, device="cuda") < held[:, None]
    pages = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    s["table"][:B][mine] = pages[:sum(-(-t // page) for t in _lens(c))]
    if c["op"] == "fork":
        # the sequences that end: a shared page, where there is one, and one of their own
        n = c["count"]
        s["src"] = (torch.randperm(n, generator=g, device="cuda") % B).to(torch.int32)
        s["dst"] = torch.randperm(n, generator=g, device="cuda").to(torch.int32) + B
        s["fork_lens"] = lens[s["src"].long()]
        s["need"] = s["fork_lens"] + c["ahead"]
        s["table"][B:, 0] = pages[-n:]
        if per > 1:
            s["table"][B:, 1] = s["table"][s["src"].long(), 0]
        s["status"] = torch.zeros(n, **i32)
        s["taken"] = torch.zeros(n, **i32)
    else:
        s["new_table"], s["new_refs"] = torch.zeros_like(s["table"]), torch.zeros(P, **i32)
        s["map"], s["used"] = torch.zeros(P, **i32), torch.zeros(1, **i32)
    named = s["table"][s["table"] >= 0].long()
    s["refs"] = torch.zeros(P, **i32).index_add_(0, named, torch.ones_like(named, dtype=torch.int32))
    return s


def _caches(s, c, normal, prefix, L, P):
    """Keys, values and scales of L layers, [layer][page][slot][head][D] and [layer][page][head][slot]; one layer without the first."""
    for x in ("k", "v"):
        rows, scale = normal(L, P, c["page"], c["Hkv"], c["D"]), None
        if c["cache"] == "e4m3":
            scale = rows.abs().amax(-1).float() / E4M3_MAX
            rows, scale = (rows / scale[..., None]).to(torch.float8_e4m3fn), scale.transpose(2, 3).contiguous()
            s[prefix + x + "_scale"] = scale[0] if c["op"] == "write" else scale
        s[prefix + x + "_cache"] = rows[0] if c["op"] == "write" else rows


# ------------------------------------------------------------------ plain forms
def _plain_attn(s):
    """Sequence by sequence, as many rows at a time as two gigabytes of scores hold."""
    c = s["case"]
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    ends = s["starts"].tolist()
    parts = [(a, b, r, min(b, r + m)) for a, b in zip(ends, ends[1:]) if b > a for m in (max(1, 2 ** 29 // (Hq * (b - a))),) for r in range(a, b, m)]
    for a, b, r0, r1 in parts:
        lo = max(a, r0 + 1 - c["window"]) if c["window"] else a
        q, k, v = (s[x][u:r1].float().transpose(0, 1) for x, u in (("q", r0), ("k", lo), ("v", lo)))
        z = (q.reshape(Hkv, -1, D) @ k.transpose(1, 2)).view(Hq, r1 - r0, -1).mul_(D ** -0.5)
        if c["softcap"]:
            z = c["softcap"] * torch.tanh(z / c["softcap"])
        r, j = torch.arange(r0, r1, device="cuda")[:, None], torch.arange(lo, r1, device="cuda")
        z.masked_fill_((j > r) | ((j <= r - c["window"]) if c["window"] else j > r), -math.inf)
        m = z.amax(-1, keepdim=True)
        e = z.sub_(m).exp_()
        total = e.sum(-1, keepdim=True)
        o = (e.view(Hkv, -1, r1 - lo) @ v).view(Hq, r1 - r0, D) / total
        s["out"][r0:r1] = o.transpose(0, 1).to(torch.bfloat16)
        s["lse"][r0:r1] = (m + total.log())[..., 0].T
    return {"out": s["out"], "lse": s["lse"]}


def _plain_write(s):
    c, m = s["case"], s["rows"]
    r = torch.arange(m, device="cuda")
    seq = torch.searchsorted(s["starts"][1:].contiguous(), r, right=True)
    pos = s["first"].long()[seq] + r - s["starts"].long()[seq]

    def finished(x, w):
        x = x[:m].float()
        if w is not None:
            x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * w.float()
        if c["rot"]:
            at = s["positions"][:, :m].long()[s["pair_axis"].long()]               # [pair][row]: each pair's position
            cos, sin = (s["rope"][:, half].gather(0, at.T)[:, None] for half in (slice(0, c["rot"] // 2), slice(c["rot"] // 2, None)))
            turned, rest = x[..., :c["rot"]], x[..., c["rot"]:]
            if c["pairs"] == "halves":
                a, b = turned.chunk(2, -1)
                x = torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
            else:
                a, b = turned[..., ::2], turned[..., 1::2]
                x = torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)
        return x

    q, k, v = finished(s["q"], s["q_norm"]), finished(s["k"], s["k_norm"]), s["v"][:m].float()
    s["out"][:m] = q.to(torch.bfloat16)
    s["k_out"][:m] = k.to(torch.bfloat16)
    slot = s["table"].long()[seq, pos // c["page"]], pos % c["page"]
    if c["cache"] == "e4m3":
        ks, vs = k.abs().amax(-1) / E4M3_MAX, v.abs().amax(-1) / E4M3_MAX
        s["k_scale"].transpose(1, 2)[slot], s["v_scale"].transpose(1, 2)[slot] = ks, vs
        k, v = (x / y[..., None] for x, y in ((k, ks), (v, vs)))
        s["k_cache"].view(torch.int8)[slot] = k.to(torch.float8_e4m3fn).view(torch.int8)
        s["v_cache"].view(torch.int8)[slot] = v.to(torch.float8_e4m3fn).view(torch.int8)
    else:
        s["k_cache"][slot], s["v_cache"][slot] = k.to(torch.bfloat16), v.to(torch.bfloat16)
    return _written(s)


def _plain_move(s, src, dst, slots, to=""):
    """Pages src of every layer's caches to pages dst of the others, the first `slots` slots of each."""
    live = (torch.arange(s["case"]["page"], device="cuda") < slots[:, None])
    moved = [("k_cache", live[..., None, None]), ("v_cache", live[..., None, None]), ("k_scale", live[:, None]), ("v_scale", live[:, None])]
    moved = [(s[x], s[to + x], m) for x, m in moved if x in s]
    for x, y, m in [(x.view(torch.int8), y.view(torch.int8), m) if x.dtype == torch.float8_e4m3fn else (x, y, m) for x, y, m in moved]:
        y[:, dst] = torch.where(m, x[:, src], y[:, dst])


def _plain_fork(s):
    c = s["case"]
    table, refs, src, dst, page = s["table"], s["refs"], s["src"].long(), s["dst"].long(), c["page"]
    entry = torch.arange(table.shape[1], device="cuda")
    count = lambda rows, by: refs.index_add_(0, rows[rows >= 0].long(), torch.full_like(rows[rows >= 0], by))
    # the sequences that ended
    count(table[dst], -1)
    # whole pages are shared, the last token's is copied
    last = (s["fork_lens"].long() - 1) // page
    rows = torch.where(entry < last[:, None], table[src], -1)
    count(rows, 1)
    tails = (refs == 0).nonzero()[:len(dst), 0]
    rows[torch.arange(len(dst), device="cuda"), last] = tails.to(torch.int32)
    refs[tails] = 1
    _plain_move(s, table[src, last].long(), tails, (s["fork_lens"] - 1) % page + 1)
    # pages for the next tokens, sequence by sequence
    lacks = (entry * page < s["need"][:, None]) & (rows < 0)
    more = (refs == 0).nonzero()[:, 0]
    more = more[:lacks.sum()]
    rows[lacks] = more.to(torch.int32)
    refs[more] = 1
    table[dst] = rows
    s["status"].zero_()
    s["taken"].zero_()
    return _forked(s)


def _plain_compact(s):
    table, refs = s["table"], s["refs"]
    used = refs > 0
    n = used.sum()
    at = torch.arange(len(refs), device="cuda")
    holes, high = (~used & (at < n)).nonzero()[:, 0], (used & (at >= n)).nonzero()[:, 0]
    new = torch.where(used, at, -1)
    new[high] = holes
    _plain_move(s, high, holes, torch.full_like(high, s["case"]["page"]))
    s["map"].copy_(new)
    s["new_table"].copy_(torch.where(table >= 0, s["map"][table.clamp(min=0).long()], table))
    s["new_refs"].zero_()[new[used]] = refs[used]
    s["used"].copy_(n)
    return _compacted(s)


def _plain_copy(s):
    _plain_move(s, s["src"].long(), s["dst"].long(), s["slots"], "to_")
    return _copied(s)


def _written(s):
    return {k: s[k] for k in ("out", "k_out", "k_cache", "v_cache", "k_scale", "v_scale") if k in s}


def _forked(s):
    return {k: s[k] for k in ("table", "refs", "status", "taken", "k_cache", "v_cache", "k_scale", "v_scale") if k in s}


def _compacted(s):
    return {k: s[k] for k in ("new_table", "new_refs", "map", "used", "k_cache", "v_cache", "k_scale", "v_scale") if k in s}


def _copied(s):
    return {k: s["to_" + k] for k in ("k_cache", "v_cache", "k_scale", "v_scale") if k in s}


# ------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    if not own:
        return {"attn": _plain_attn, "write": _plain_write, "fork": _plain_fork, "compact": _plain_compact, "copy": _plain_copy}[c["op"]](s)
    import paper_2412_01447_amd as pld
    if c["op"] == "attn":
        pld.pld_prompt_attn(s["q"], s["k"], s["v"], s["starts"], s["out"], lse=s["lse"], softcap=c["softcap"], window=c["window"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "write":
        pld.pld_cache_write_packed(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["starts"], s["first"], s["out"], k_out=s["k_out"],
                                   k_scale=s.get("k_scale"), v_scale=s.get("v_scale"), q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS, rope=s["rope"],
                                   rope_pairs=pld.PLD_ROPE_HALVES if c["pairs"] == "halves" else pld.PLD_ROPE_NEIGHBOURS, positions=s["positions"],
                                   pair_axis=s["pair_axis"])
        return _written(s)
    from paper_2412_01447_amd.cache import PagePool
    if "pool" not in s:
        layers = lambda prefix: [list(s[prefix + x].unbind(0)) if prefix + x in s else None for x in ("k_cache", "v_cache", "k_scale", "v_scale")]
        s["pool"] = PagePool(*layers(""), table=s.get("table"), refs=s.get("refs"))
        if c["op"] == "copy":
            s["to_pool"] = PagePool(*layers("to_"))
    if c["op"] == "fork":
        s["pool"].free(s["dst"])
        s["pool"].fork(s["src"], s["dst"], s["fork_lens"], s["status"])
        s["pool"].take(s["dst"], s["need"], s["taken"])
        return _forked(s)
    if c["op"] == "compact":
        s["pool"].compact(s["map"], s["used"], table_out=s["new_table"], refs_out=s["new_refs"])
        return _compacted(s)
    s["to_pool"].copy_from(s["pool"], s["src"], s["dst"], s["slots"])
    return _copied(s)


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """What run() returns, one sequence (and head) at a time in 64 bits; pages, one table entry at a time on the host."""
    c, s = case, prepare(case, seed)
    f64, page = torch.float64, case["page"]
    if c["op"] == "attn":
        r = {"out": s["out"].to(f64), "lse": s["lse"].to(f64)}
        G, ends = c["Hq"] // c["Hkv"], s["starts"].tolist()
        for a, b in zip(ends, ends[1:]):
            step = max(1, 2 ** 28 // (G * (b - a)))
            for h in range(c["Hkv"]):
                k, v = s["k"][a:b, h].to(f64), s["v"][a:b, h].to(f64)
                for x in range(a, b, step):
                    y = min(b, x + step)
                    z = torch.tensordot(s["q"][x:y, h * G:(h + 1) * G].to(f64), k[:y - a], ([2], [1])) / math.sqrt(c["D"])   # [rows][G][keys]
                    if c["softcap"]:
                        z = c["softcap"] * torch.tanh(z / c["softcap"])
                    ahead = torch.arange(a, y, device="cuda") - torch.arange(x, y, device="cuda")[:, None, None]
                    z.masked_fill_((ahead > 0) | (ahead <= -(c["window"] or b - a)), -math.inf)
                    r["lse"][x:y, h * G:(h + 1) * G] = z.logsumexp(-1)
                    r["out"][x:y, h * G:(h + 1) * G] = torch.tensordot(z.softmax(-1), v[:y - a], 1)
        return r
    if c["op"] == "write":
        r = {k: v.to(f64) for k, v in _written(s).items()}
        starts, first = s["starts"].tolist(), s["first"].tolist()
        for b in range(c["B"]):
            rows = torch.arange(starts[b], starts[b + 1], device="cuda")
            at = first[b] + rows - starts[b]
            slot = s["table"][b].long()[at // page], at % page
            for x, w in (("q", s["q_norm"]), ("k", s["k_norm"]), ("v", None)):
                y = s[x][rows].to(f64)
                if w is not None:
                    y = y / (y.pow(2).sum(-1, keepdim=True) / c["D"] + EPS).sqrt() * w.to(f64)
                if x != "v" and c["rot"]:
                    half = c["rot"] // 2
                    where = s["positions"].long()[:, rows]
                    by = [s["rope"][where[a], t].to(f64) + 1j * s["rope"][where[a], half + t].to(f64) for t, a in enumerate(s["pair_axis"].tolist())]
                    head = y[..., :2 * half]
                    pair = head.unflatten(-1, (2, -1)).transpose(-1, -2) if c["pairs"] == "halves" else head.unflatten(-1, (-1, 2))
                    pair = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * torch.stack(by, -1)[:, None])
                    y = torch.cat([(pair.transpose(-1, -2) if c["pairs"] == "halves" else pair).flatten(-2), y[..., 2 * half:]], -1)
                if x == "q":
                    r["out"][rows] = y
                    continue
                if x == "k":
                    r["k_out"][rows] = y
                if c["cache"] == "e4m3":
                    scale = y.abs().amax(-1) / E4M3_MAX
                    r[x + "_scale"][slot[0], :, slot[1]] = scale
                    y = y / scale[..., None]
                    step = torch.exp2(y.abs().clamp(min=2.0 ** -6).log2().floor() - 3)     # three bits behind the leading one
                    y = (y / step).round() * step
                r[x + "_cache"][slot] = y
        return r
    names = [x for x in ("k_cache", "v_cache", "k_scale", "v_scale") if x in s]
    to = "to_" if c["op"] == "copy" else ""
    r = {x: s[to + x].clone() for x in names}

    def move(i, j, slots):
        for x in names:
            if x.endswith("cache"):
                r[x][:, j, :slots] = s[x][:, i, :slots]
            else:
                r[x][:, j, :, :slots] = s[x][:, i, :, :slots]

    if c["op"] == "copy":
        for i, j, m in zip(s["src"].tolist(), s["dst"].tolist(), s["slots"].tolist()):
            move(i, j, m)
        return r
    table, refs = s["table"].tolist(), s["refs"].tolist()
    if c["op"] == "fork":
        for j in s["dst"].tolist():
            for p, x in enumerate(table[j]):
                if x >= 0:
                    refs[x] -= 1
                table[j][p] = -1
        forks, lens, tails = list(zip(s["src"].tolist(), s["dst"].tolist())), s["fork_lens"].tolist(), []
        for (i, j), t in zip(forks, lens):
            for p in range((t - 1) // page):
                table[j][p] = table[i][p]
                refs[table[i][p]] += 1
        free = (x for x, n in enumerate(list(refs)) if n == 0)
        for (i, j), t in zip(forks, lens):
            p, x = (t - 1) // page, next(free)
            table[j][p], refs[x] = x, 1
            move(table[i][p], x, t - p * page)
        for (_, j), need in zip(forks, s["need"].tolist()):
            for p in range(-(-need // page)):
                if table[j][p] < 0:
                    table[j][p] = x = next(free)
                    refs[x] = 1
        return dict(r, table=torch.tensor(table, dtype=torch.int32), refs=torch.tensor(refs, dtype=torch.int32), status=s["status"], taken=s["taken"])
    n = sum(x > 0 for x in refs)
    new, new_refs, hole = [-1] * len(refs), [0] * len(refs), 0
    for x, k in enumerate(refs):
        if k == 0:
            continue
        new[x] = x
        if x >= n:
            while refs[hole]:
                hole += 1
            new[x], hole = hole, hole + 1
            move(x, new[x], page)
        new_refs[new[x]] = k
    table = [[new[x] if x >= 0 else x for x in row] for row in table]
    ints = {k: torch.tensor(v, dtype=torch.int32) for k, v in (("new_table", table), ("new_refs", new_refs), ("map", new), ("used", [n]))}
    return dict(r, **ints)
