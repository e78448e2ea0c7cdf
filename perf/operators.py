"""The model side of a verification pass: the operators' cases, their plain forms and their values in 64 bits.

Verifying a draft of K tokens runs the target model over K+1 rows per sequence: row i holds position
lens[b]-1+i (the last committed token, then the draft), and rows i <= draft_len[b] exist.  Per layer the
rows' keys and values join a paged cache (heads normed, rotated, quantised as they are written), the rows
attend to the cache, and the heads that rank the next drafting step give the weights of one row.  After
the last layer the emitted tokens' log probabilities go out with their alternatives.

  write     x / sqrt(mean(x^2) + eps) * w per head, the pairs of the first `rot` elements turned by the
            position's angle; q back to the program, k and v to their page slots (e4m3: one scale a row and head)
  attend    softmax over keys p - window < j <= p of cap * tanh(q.k * scale / cap), times v; with its log sum
  rows      exp(score - log sum) of the chosen heads at row row[b], over keys 0..position
  logprobs  log softmax(z / tau) at the given tokens, its entropy, and its largest entries, lowest id first
"""
import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0


# ------------------------------------------------------------------ cases
def _case(name=None, *, op, B, n, T=0, ragged=0.0, Hq=0, Hkv=0, D=0, page=0, cache="", rot=0, pairs="halves",
          norm=False, softcap=0.0, window=0, R=0, V=0, logits="", top=0, tau=1.0, masked=0.0):
    """n: rows a sequence (K + 1); T: the longest committed length, and ragged: the shortest is (1 - ragged) T and every third
    draft is cut; page: token slots a page; pairs: the elements turned together, d and d + rot/2 ("halves") or 2d and 2d + 1
    ("neighbours"); R: heads whose weights go out; masked: share of the vocabulary at minus infinity in every second row."""
    c = dict(op=op, B=B, n=n, T=T, ragged=ragged, Hq=Hq, Hkv=Hkv, D=D, page=page, cache=cache, rot=rot, pairs=pairs, norm=norm,
             softcap=softcap, window=window, R=R, V=V, logits=logits, top=top, tau=tau, masked=masked)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # one user's next token without a draft: launch and latency
        _case("write_b1_n1", op="write", B=1, n=1, T=1024, Hq=32, Hkv=8, D=128, page=16, cache="bf16", rot=128, norm=True),
        # the largest batch's verification rows into a quantised cache
        _case("write_b64_n17_e4m3", op="write", B=64, n=17, T=400, ragged=0.5, Hq=64, Hkv=8, D=128, page=64, cache="e4m3", rot=128, norm=True),
        # prompts read in chunks: many rows a sequence, half of each head turned, neighbouring pairs, no norms
        _case("write_b4_n2048_chunk", op="write", B=4, n=2048, T=600, Hq=32, Hkv=8, D=128, page=32, cache="bf16", rot=64, pairs="neighbours"),
        # one user's next token without a draft
        _case("attend_b1_t1024_n1", op="attend", B=1, n=1, T=1024, Hq=32, Hkv=8, D=128, page=16, cache="bf16"),
        # a small serving batch of ragged lengths with ten drafted tokens
        _case("attend_b8_t4096_n11", op="attend", B=8, n=11, T=4096, ragged=0.6, Hq=32, Hkv=8, D=128, page=16, cache="bf16"),
        # capped scores in a window, narrow heads, odd lengths, few rows
        _case("attend_b12_t3333_window", op="attend", B=12, n=8, T=3333, ragged=0.7, Hq=24, Hkv=4, D=64, page=32, cache="bf16", softcap=30.0, window=1000),
        # the largest batch over a quantised cache
        _case("attend_b64_t16384_e4m3", op="attend", B=64, n=17, T=16384, ragged=0.2, Hq=64, Hkv=8, D=128, page=64, cache="e4m3"),
        # few sequences with the longest contexts and drafts
        _case("attend_b4_t131072_n33", op="attend", B=4, n=33, T=131072, Hq=32, Hkv=8, D=128, page=64, cache="bf16"),
        # one user's selected heads of one layer, for the next step's ranking
        _case("rows_b1_t1024_r8", op="rows", B=1, n=71, T=1024, Hq=32, Hkv=32, D=128, page=16, cache="bf16", R=8),
        # all heads of a layer for a serving batch
        _case("rows_b32_t8192_r40", op="rows", B=32, n=17, T=8192, ragged=0.25, Hq=40, Hkv=8, D=128, page=64, cache="bf16", R=40),
        # one user's step: eleven rows, five alternatives each
        _case("logprobs_b1_n11_v32000", op="logprobs", B=1, n=11, V=32000, logits="f32", top=5),
        # the largest batch and vocabulary, twenty alternatives, part of the rows under a grammar's mask
        _case("logprobs_b64_n17_v128256", op="logprobs", B=64, n=17, ragged=0.5, V=128256, logits="bf16", top=20, tau=0.8, masked=0.5),
    ]


def _spread(rng, lo, hi):
    """A whole number, its logarithm uniform over [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["write", "attend", "attend", "rows", "logprobs"])
        B, ragged = _spread(rng, 1, 64), rng.choice([0.0, round(rng.uniform(0.1, 0.9), 2)])
        if op == "logprobs":
            c = _case(op=op, B=B, n=_spread(rng, 1, 71), ragged=ragged, V=_spread(rng, 1000, 160000), logits=rng.choice(["f32", "bf16"]),
                      top=rng.choice([0, 1, 5, 20, rng.randint(2, 32)]), tau=rng.choice([1.0, 0.7, 1.3]), masked=rng.choice([0.0, 0.9]))
        else:
            heads, group = rng.choice([1, 2, 4, 8, 8, 16, 32]), rng.choice([1, 2, 4, 5, 6, 7, 8, 12, 16])
            c = dict(B=B, ragged=ragged, Hq=heads * group, Hkv=heads, D=rng.choice([64, 128, 128, 256]), page=rng.choice([16, 32, 64, 128]),
                     cache=rng.choice(["bf16", "e4m3"]))
            if op == "write":
                c = _case(op=op, n=_spread(rng, 1, 3000), T=_spread(rng, 1, 600), rot=rng.choice([c["D"], c["D"] // 2, 0]),
                          pairs=rng.choice(["halves", "neighbours"]), norm=rng.random() < 0.5, **c)
            else:
                cap, window = rng.choice([(0.0, 0), (0.0, 0), (30.0, 0), (0.0, _spread(rng, 16, 20000)), (50.0, _spread(rng, 16, 20000))])
                c = _case(op=op, n=_spread(rng, 1, 71), T=_spread(rng, 1, 131072), softcap=cap, window=window,
                          R=rng.randint(1, c["Hq"]) if op == "rows" else 0, **c)
            if c["Hq"] > 128:
                continue
        w, most = work(c), _most[op]
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"] and _held(c) <= 3.2e9:
            return c


# ------------------------------------------------------------------ what a pass cannot do without
def _lens(c):
    B, T = c["B"], c["T"]
    return [T - int(c["ragged"] * (T - 1) * b / max(1, B - 1)) for b in range(B)]


def _counts(c):
    """Rows of each sequence that exist."""
    return [c["n"] if b % 3 != 1 or not c["ragged"] else 1 + (c["n"] - 1) // 2 for b in range(c["B"])]


def _pages(c):
    """Pages a sequence's block table holds."""
    return -(-(c["T"] + c["n"]) // c["page"])


def _held(c):
    """Bytes of the cache, or of the logits."""
    if c["op"] == "logprobs":
        return c["B"] * c["n"] * c["V"] * (4 if c["logits"] == "f32" else 2)
    return 2 * c["B"] * _pages(c) * c["page"] * c["Hkv"] * c["D"] * (2 if c["cache"] == "bf16" else 1)


def work(case):
    c = case
    lens, counts = _lens(c) if c["T"] else [0] * c["B"], _counts(c)
    rows = sum(counts)
    if c["op"] == "logprobs":
        return {"bytes": rows * (c["V"] * (4 if c["logits"] == "f32" else 2) + 12 + 8 * c["top"]), "flops": rows * c["V"] * 5}
    D, Hq, Hkv = c["D"], c["Hq"], c["Hkv"]
    row = D * 2 if c["cache"] == "bf16" else D + 4              # one head's key or value of one token in the cache
    if c["op"] == "write":
        table = len({t - 1 + i for t, m in zip(lens, counts) for i in range(m)}) * c["rot"] * 4
        return {"bytes": rows * (4 * D * Hq + 4 * D * Hkv + 2 * row * Hkv) + table, "flops": rows * D * (Hq + 2 * Hkv) * 8}
    keys = lambda t, p: min(p + 1, c["window"]) if c["window"] else p + 1          # keys that position p sees
    if c["op"] == "rows":
        b = f = 0
        for t, m in zip(lens, counts):
            p = t - 1 + (m - 1) // 2
            b += keys(t, p) * row * min(Hkv, c["R"]) + (p + 1) * 4 * c["R"] + c["R"] * (2 * D + 4)
            f += keys(t, p) * 2 * D * c["R"]
        return {"bytes": b, "flops": f}
    b = sum((min(t - 1 + m, c["window"] + m - 1) if c["window"] else t - 1 + m) * 2 * row * Hkv for t, m in zip(lens, counts))
    f = sum(4 * D * Hq * sum(keys(t, t - 1 + i) for i in range(m)) for t, m in zip(lens, counts))
    return {"bytes": b + rows * Hq * (4 * D + 4), "flops": f}


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
    mix = torch.randperm(c["B"], generator=g, device="cuda")                      # which sequence has which length
    s = dict(case=c, count=torch.tensor(_counts(c), **i32)[mix])
    B, n = c["B"], c["n"]
    if c["op"] == "logprobs":
        V, N = c["V"], c["top"]
        z = normal(B, n, V).mul_(2.5)
        s["tokens"] = torch.randint(0, V, (B, n), generator=g, **i32)
        if c["masked"]:
            allowed = torch.rand(V, generator=g, device="cuda") >= c["masked"]
            allowed[s["tokens"].long()] = True
            z[:, ::2] = torch.where(allowed, z[:, ::2], -math.inf)
        s["logits"] = z.float() if c["logits"] == "f32" else z
        if c["logits"] == "f32":
            s["logits"] += torch.rand(B, n, V, generator=g, device="cuda").mul_(0.01)
        # the emitted tokens are mostly the likely ones
        s["logits"].scatter_(2, s["tokens"].long()[..., None], normal(B, n, 1).mul_(3).add_(9).to(z.dtype).to(s["logits"].dtype))
        s["logprob"] = torch.zeros(B, n, device="cuda")
        s["entropy"] = torch.zeros(B, n, device="cuda")
        s["top_ids"] = torch.zeros(B, n, N, **i32)
        s["top_logprobs"] = torch.zeros(B, n, N, device="cuda")
        return s
    Hq, Hkv, D, page = c["Hq"], c["Hkv"], c["D"], c["page"]
    s["lens"] = torch.tensor(_lens(c), **i32)[mix]
    s["draft_len"] = s["count"] - 1
    P = B * _pages(c)
    s["table"] = torch.randperm(P, generator=g, device="cuda").to(torch.int32).view(B, -1)
    s["k_cache"], s["v_cache"] = normal(P, page, Hkv, D), normal(P, page, Hkv, D)
    if c["cache"] == "e4m3":
        for x in ("k", "v"):
            rows = s[x + "_cache"].float()
            scale = rows.abs().amax(-1) / E4M3_MAX
            s[x + "_cache"] = (rows / scale[..., None]).to(torch.float8_e4m3fn)
            s[x + "_scale"] = scale.permute(0, 2, 1).contiguous()                  # [page][head][slot]
    if c["op"] == "write":
        # one projection's output: q, k and v of a row side by side
        qkv = normal(B, n, (Hq + 2 * Hkv) * D)
        q, k, v = qkv.split([Hq * D, Hkv * D, Hkv * D], -1)
        s["q"], s["k"], s["v"] = q.unflatten(-1, (Hq, D)), k.unflatten(-1, (Hkv, D)), v.unflatten(-1, (Hkv, D))
        s["q_out"] = torch.zeros(B, n, Hq, D, dtype=torch.bfloat16, device="cuda")
        s["q_norm"] = s["k_norm"] = s["rope"] = None
        if c["norm"]:
            s["q_norm"], s["k_norm"] = normal(D).mul_(0.1).add_(1), normal(D).mul_(0.1).add_(1)
        if c["rot"]:
            freq = 500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device="cuda") / c["rot"])
            angle = torch.arange(c["T"] + n, dtype=torch.float64, device="cuda")[:, None] * freq
            s["rope"] = torch.cat([angle.cos(), angle.sin()], -1).float()
        return s
    s["q"] = normal(B, n, Hq, D).mul_(2)
    if c["op"] == "attend":
        s["out"] = torch.zeros(B, n, Hq, D, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros(B, n, Hq, device="cuda")
        return s
    s["row"] = s["draft_len"] // 2
    s["heads"] = torch.randperm(Hq, generator=g, device="cuda")[:c["R"]].to(torch.int32).sort()[0]
    s["lse"] = torch.zeros(B, n, Hq, device="cuda")
    s["attn"] = torch.zeros(B, c["R"], c["T"] + n, device="cuda")
    at = torch.arange(B, device="cuda")
    s["lse"][at, s["row"].long()] = _scores(s, s["q"][at, s["row"].long()][:, None], s["row"][:, None]).logsumexp(-1)[:, :, 0]
    return s


# ------------------------------------------------------------------ plain forms
def _dense(s, x):
    """The cache's keys or values in order of position: fp32 [B][Hkv][slots][D]."""
    t = s["table"].long()
    rows = s[x + "_cache"][t].float()                                              # [B][pages][page][Hkv][D]
    if x + "_scale" in s:
        rows = rows * s[x + "_scale"][t].transpose(2, 3)[..., None]
    return rows.flatten(1, 2).transpose(1, 2)


def _scores(s, q, i):
    """Scores of the query rows q [B][m][Hq][D] at rows i [B][m], minus infinity where a key is not seen: [B][Hq][m][slots]."""
    c, k = s["case"], _dense(s, "k")
    B, m, Hq, D = q.shape
    rows = q.float().transpose(1, 2).reshape(B, c["Hkv"], -1, D)                   # a key head's query heads, row by row
    z = (rows @ k.transpose(2, 3)).view(B, Hq, m, -1) * D ** -0.5
    if c["softcap"]:
        z = c["softcap"] * torch.tanh(z / c["softcap"])
    p, j = (s["lens"][:, None] - 1 + i)[:, None, :, None], torch.arange(z.shape[-1], device="cuda")
    seen = j <= p
    if c["window"]:
        seen = seen & (j > p - c["window"])
    return torch.where(seen, z, -math.inf)


def _plain_write(s):
    c = s["case"]
    B, n, D = c["B"], c["n"], c["D"]
    i = torch.arange(n, device="cuda")
    pos, live = (s["lens"][:, None] - 1 + i).long(), (i <= s["draft_len"][:, None])[..., None, None]

    def finished(x, w):
        x = x.float()
        if w is not None:
            x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * w.float()
        if c["rot"]:
            cos, sin = s["rope"][pos][:, :, None].chunk(2, -1)
            turned, rest = x[..., :c["rot"]], x[..., c["rot"]:]
            if c["pairs"] == "halves":
                a, b = turned.chunk(2, -1)
                x = torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
            else:
                a, b = turned[..., ::2], turned[..., 1::2]
                x = torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)
        return x

    q = finished(s["q"], s["q_norm"]).to(torch.bfloat16)
    s["q_out"].copy_(torch.where(live, q, s["q_out"]))
    slot = s["table"].long().gather(1, pos // c["page"]), pos % c["page"]
    for x, rows in (("k", finished(s["k"], s["k_norm"])), ("v", s["v"].float())):
        if c["cache"] == "e4m3":
            scale = rows.abs().amax(-1) / E4M3_MAX
            rows = rows / scale[..., None]
            by_slot = s[x + "_scale"].transpose(1, 2)
            by_slot[slot] = torch.where(live[..., 0], scale, by_slot[slot])
        cache = s[x + "_cache"]
        whole = cache.view(torch.int8) if c["cache"] == "e4m3" else cache           # rows that do not exist keep their bits
        new = rows.to(cache.dtype)
        whole[slot] = torch.where(live, new.view(whole.dtype), whole[slot])
    return _written(s)


def _plain_attend(s):
    c = s["case"]
    B, n, Hq, D = c["B"], c["n"], c["Hq"], c["D"]
    i = torch.arange(n, device="cuda").expand(B, n)
    z = _scores(s, s["q"], i)
    m = z.amax(-1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(-1, keepdim=True)
    o = (e / total).view(B, c["Hkv"], -1, z.shape[-1]) @ _dense(s, "v")
    live = i <= s["draft_len"][:, None]
    s["out"].copy_(torch.where(live[..., None, None], o.view(B, Hq, n, D).transpose(1, 2).to(torch.bfloat16), s["out"]))
    s["lse"].copy_(torch.where(live[..., None], (m + total.log())[..., 0].transpose(1, 2), s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


def _plain_rows(s):
    at, row, heads = torch.arange(s["case"]["B"], device="cuda"), s["row"].long(), s["heads"].long()
    z = _scores(s, s["q"][at, row][:, None], s["row"][:, None])[:, heads, 0]        # [B][R][slots]
    w = (z - s["lse"][at, row][:, heads, None]).exp()[..., :s["attn"].shape[-1]]
    p = (s["lens"] - 1 + s["row"])[:, None, None]
    s["attn"].copy_(torch.where(torch.arange(w.shape[-1], device="cuda") <= p, w, s["attn"]))
    return {"attn": s["attn"]}


def _plain_logprobs(s):
    c = s["case"]
    z = s["logits"].float() / c["tau"]
    m = z.amax(-1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(-1, keepdim=True)
    at = z.gather(-1, s["tokens"].long()[..., None])
    live = torch.arange(c["n"], device="cuda") < s["count"][:, None]
    s["logprob"].copy_(torch.where(live, ((at - m) - total.log())[..., 0], s["logprob"]))
    weighted = torch.where(e > 0, e * (z - m), 0).sum(-1, keepdim=True)
    s["entropy"].copy_(torch.where(live, (total.log() - weighted / total)[..., 0], s["entropy"]))
    if c["top"]:
        # one whole number an entry, larger for a larger logit and, among equals, for a lower id
        bits = (s["logits"].float() + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() << 32
        ids = (order | (0xffffffff - torch.arange(c["V"], device="cuda"))).topk(c["top"], -1)[0]
        ids = 0xffffffff - (ids & 0xffffffff)
        s["top_ids"].copy_(torch.where(live[..., None], ids.to(torch.int32), s["top_ids"]))
        s["top_logprobs"].copy_(torch.where(live[..., None], (z.gather(-1, ids) - m) - total.log(), s["top_logprobs"]))
    return {k: s[k] for k in ("logprob", "entropy", "top_ids", "top_logprobs")}


def _written(s):
    return {k: s[k] for k in ("q_out", "k_cache", "v_cache", "k_scale", "v_scale") if k in s}


# ------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    if not own:
        return {"write": _plain_write, "attend": _plain_attend, "rows": _plain_rows, "logprobs": _plain_logprobs}[c["op"]](s)
    import paper_2412_01447_amd as pld
    if c["op"] == "write":
        pld.pld_cache_write(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["q_out"], draft_len=s["draft_len"],
                            k_scale=s.get("k_scale"), v_scale=s.get("v_scale"), q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS,
                            rope=s["rope"], rope_pairs=pld.PLD_ROPE_HALVES if c["pairs"] == "halves" else pld.PLD_ROPE_NEIGHBOURS)
        return _written(s)
    if c["op"] == "attend":
        if "workspace" not in s:
            need = pld.pld_cache_attn_workspace_bytes(c["B"], c["n"], c["Hq"], c["Hkv"], c["D"])
            s["workspace"] = torch.zeros(need, dtype=torch.uint8, device="cuda")
        pld.pld_cache_attn(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["out"], s["workspace"], draft_len=s["draft_len"],
                           k_scale=s.get("k_scale"), v_scale=s.get("v_scale"), lse=s["lse"], softcap=c["softcap"], window=c["window"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "rows":
        pld.pld_cache_attn_rows(s["q"], s["k_cache"], s["table"], s["lens"], s["row"], s["heads"], s["lse"], s["attn"],
                                k_scale=s.get("k_scale"), softcap=c["softcap"], window=c["window"])
        return {"attn": s["attn"]}
    if "workspace" not in s:
        need = pld.pld_token_logprobs_workspace_bytes(c["B"], c["n"], c["V"], pld.PLD_F32 if c["logits"] == "f32" else pld.PLD_BF16, c["top"])
        s["workspace"] = torch.zeros(need, dtype=torch.uint8, device="cuda")
    top = c["top"] > 0
    pld.pld_token_logprobs(s["logits"], s["tokens"], s["logprob"], s["workspace"], count=s["count"], temperature=c["tau"], entropy=s["entropy"],
                           top_ids=s["top_ids"] if top else None, top_logprobs=s["top_logprobs"] if top else None)
    return {k: s[k] for k in ("logprob", "entropy", "top_ids", "top_logprobs")}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """What run() returns, one sequence at a time in 64 bits."""
    c, s = case, prepare(case, seed)
    f64 = torch.float64
    count, B, n = s["count"].tolist(), c["B"], c["n"]
    if c["op"] == "logprobs":
        out = {k: s[k].to(f64) for k in ("logprob", "entropy", "top_logprobs")}
        ids = s["top_ids"].clone()
        for b, m in enumerate(count):
            lp = (s["logits"][b, :m].to(f64) / c["tau"]).log_softmax(-1)
            out["logprob"][b, :m] = lp.gather(-1, s["tokens"][b, :m, None].long())[..., 0]
            out["entropy"][b, :m] = torch.special.entr(lp.exp()).sum(-1)
            if c["top"]:
                first = s["logits"][b, :m].sort(dim=-1, descending=True, stable=True)[1][..., :c["top"]]
                ids[b, :m] = first.to(torch.int32)
                out["top_logprobs"][b, :m] = lp.gather(-1, first)
        return dict(out, top_ids=ids)
    lens, page = s["lens"].tolist(), c["page"]
    if c["op"] == "write":
        r = {k: s[k].to(f64) for k in ("q_out", "k_cache", "v_cache", "k_scale", "v_scale") if k in s}
        for b, m in enumerate(count):
            at = torch.arange(lens[b] - 1, lens[b] - 1 + m, device="cuda")
            slot = s["table"][b].long()[at // page], at % page
            for x, w in (("q", s["q_norm"]), ("k", s["k_norm"]), ("v", None)):
                y = s[x][b, :m].to(f64)
                if w is not None:
                    y = y / (y.pow(2).sum(-1, keepdim=True) / c["D"] + EPS).sqrt() * w.to(f64)
                if x != "v" and c["rot"]:
                    t = s["rope"][at].to(f64)[:, None]
                    turn = torch.complex(t[..., :c["rot"] // 2], t[..., c["rot"] // 2:])
                    y, head = y.clone(), y[..., :c["rot"]]
                    pair = head.unflatten(-1, (2, -1)).transpose(-1, -2) if c["pairs"] == "halves" else head.unflatten(-1, (-1, 2))
                    pair = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
                    y[..., :c["rot"]] = (pair.transpose(-1, -2) if c["pairs"] == "halves" else pair).flatten(-2)
                if x == "q":
                    r["q_out"][b, :m] = y
                elif c["cache"] == "bf16":
                    r[x + "_cache"][slot] = y
                else:
                    scale = y.abs().amax(-1) / E4M3_MAX
                    y = y / scale[..., None]
                    step = torch.exp2(y.abs().clamp(min=2.0 ** -6).log2().floor() - 3)     # three bits behind the leading one
                    r[x + "_cache"][slot] = (y / step).round() * step
                    r[x + "_scale"][slot[0], :, slot[1]] = scale
        return r
    r = {"out": s["out"].to(f64), "lse": s["lse"].to(f64)} if c["op"] == "attend" else {"attn": s["attn"].to(f64)}
    G = c["Hq"] // c["Hkv"]
    for b, m in enumerate(count):
        i = [int(s["row"][b])] if c["op"] == "rows" else list(range(m))
        hi = lens[b] + i[-1]
        lo = max(0, lens[b] + i[0] - c["window"]) if c["window"] else 0
        at = torch.arange(lo, hi, device="cuda")
        slot = s["table"][b].long()[at // page], at % page
        p = torch.tensor([lens[b] - 1 + x for x in i], device="cuda")[:, None, None]
        hidden = at > p
        if c["window"]:
            hidden |= at <= p - c["window"]
        for h in range(c["Hkv"]):
            k, v = (s[x + "_cache"][slot[0], slot[1], h].to(f64) for x in "kv")
            if c["cache"] == "e4m3":
                k, v = (y * s[x + "_scale"][slot[0], h, slot[1]].to(f64)[:, None] for x, y in (("k", k), ("v", v)))
            z = (s["q"][b, i, h * G:(h + 1) * G].to(f64) @ k.T.contiguous()) / math.sqrt(c["D"])     # [rows][G][keys]
            if c["softcap"]:
                z = c["softcap"] * torch.tanh(z / c["softcap"])
            z.masked_fill_(hidden, -math.inf)
            if c["op"] == "attend":
                r["out"][b, :m, h * G:(h + 1) * G] = z.softmax(-1) @ v
                r["lse"][b, :m, h * G:(h + 1) * G] = z.logsumexp(-1)
            else:
                for a, head in enumerate(s["heads"].tolist()):
                    if head // G == h:
                        r["attn"][b, a, lo:hi] = (z[0, head - h * G] - s["lse"][b, i[0], head].to(f64)).exp()
    return r
