"""include/pld_prompt.h and its calls' host checks (CPU only; no kernel is launched here)."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

import paper_2412_01447_amd as pld
from paper_2412_01447_amd import cache
from paper_2412_01447_amd.cache import PagePool
from test_model_abi import BAD_CACHES, MIS, NULL, Q8, F, P, _cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "pld_prompt.h")
no_gpu = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="placeholder pointers are only used where no GPU is visible")


def _text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_declared_calls_are_exported_and_bound():
    names = sorted(set(re.findall(r"\b(pld_\w+)\s*\(", _text())))
    assert names == ["pld_cache_write_packed", "pld_pages_compact", "pld_pages_copy", "pld_pages_fork",
                     "pld_pages_free", "pld_pages_take", "pld_pages_workspace_bytes", "pld_prompt_attn",
                     "pld_prompt_version"]
    for n in names:
        assert hasattr(pld, n) and n in pld.__all__
        args = re.search(r"\b%s\s*\(([^)]*)\)" % n, _text()).group(1).strip()
        assert len(pld._SIGNATURES[n][0]) == (0 if args == "void" else args.count(",") + 1), n
        assert len(getattr(pld._load(), n).argtypes) == len(pld._SIGNATURES[n][0])
    for name, value in re.findall(r"#define (PLD_MAX_\w+) (\d+)", open(HEADER).read()):
        assert getattr(pld, name) == int(value), name
    m = re.search(r"#define PLD_PROMPT_ABI_VERSION (\d+)", open(HEADER).read())
    assert pld.pld_prompt_version() == int(m.group(1))


def test_struct_matches_the_header(tmp_path):
    fields = [f for f, _ in pld._Pool._fields_]
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "pld_prompt.h"\nint main(void) {\n' + "".join(
        f'printf("%zu\\n", offsetof(pld_pool, {f}));\n' for f in fields) + 'printf("%zu\\n", sizeof(pld_pool));\nreturn 0; }\n')
    for cc, std in (("gcc", "-std=c99"), ("g++", "-std=c++17")):
        subprocess.run([cc, std, "-Wall", "-Wextra", "-pedantic", "-Werror", "-x", "c" if cc == "gcc" else "c++",
                        "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "t")], check=True)
        out = subprocess.run([str(tmp_path / "t")], check=True, capture_output=True, text=True).stdout.split()
        assert [int(x) for x in out] == [getattr(pld._Pool, f).offset for f in fields] + [ctypes.sizeof(pld._Pool)]


WRITE = dict(q=F, qr=256, k=F, kr=128, v=F, vr=128, qn=NULL, kn=NULL, eps=1e-6, rope=F, rs=64, n_pos=9, rot=64, pairs=0,
             pos=F, axes=3, as_=5, pa=F, starts=F, first=F, B=2, N=5, Hq=4, out=F, orow=256, ko=F, kor=128, stream=NULL)
ATTN = dict(q=F, qr=256, k=F, kr=128, v=P(0x2000), vr=128, starts=F, B=2, N=5, Hq=4, heads=2, D=64, scale=1.0, cap=0.0, window=0,
            out=P(0x9000), orow=256, lse=F, stream=NULL)


@no_gpu
def test_write_refusals():
    fn, c = pld._load().pld_cache_write_packed, _cache()

    def status(cache=c, **kw):
        return fn(cache, *{**WRITE, **kw}.values())

    for kw, want in BAD_CACHES:
        assert status(_cache(**kw)) == want, kw
    for name in ("q", "k", "v", "starts", "first", "out"):
        assert status(**{name: NULL}) == 1, name
    for bad in (dict(B=0), dict(B=65536), dict(N=0), dict(N=(1 << 24) + 1), dict(Hq=3), dict(Hq=0), dict(Hq=4098), dict(qr=255),
                dict(kr=127), dict(vr=100), dict(kor=120), dict(eps=-1.0), dict(eps=math.nan), dict(pairs=2), dict(n_pos=0),
                dict(rot=12), dict(rot=72), dict(rot=0), dict(rs=60), dict(axes=0), dict(axes=5), dict(as_=4),
                dict(q=P(0x8000), out=P(0x8000), orow=264), dict(k=P(0x8000), ko=P(0x8000), kor=136)):
        assert status(**bad) == 1, bad
    for bad in (dict(q=MIS), dict(k=MIS), dict(v=MIS), dict(out=MIS), dict(ko=MIS), dict(qr=260), dict(qn=MIS), dict(kn=MIS),
                dict(rope=MIS), dict(rs=66), dict(pa=MIS), dict(starts=P(0x1001)), dict(first=P(0x1002)), dict(pos=P(0x1001))):
        assert status(**bad) == 2, bad


@no_gpu
def test_write_refuses_outputs_over_inputs():
    fn, c = pld._load().pld_cache_write_packed, _cache()
    apart = {**WRITE, **dict(k=P(0x20000), v=P(0x30000), out=P(0x40000), ko=P(0x50000))}
    for bad in (dict(out=P(0x20000)), dict(out=P(0x30000)), dict(ko=WRITE["q"]), dict(ko=P(0x30000)), dict(ko=P(0x40000))):
        assert fn(c, *{**apart, **bad}.values()) == 1, bad


@no_gpu
def test_attn_refusals():
    fn = pld._load().pld_prompt_attn

    def status(**kw):
        return fn(*{**ATTN, **kw}.values())

    for name in ("q", "k", "v", "starts", "out"):
        assert status(**{name: NULL}) == 1, name
    for bad in (dict(B=0), dict(B=65536), dict(N=0), dict(N=(1 << 24) + 1), dict(Hq=5), dict(Hq=0), dict(Hq=4098), dict(heads=0),
                dict(heads=1025, Hq=1025), dict(D=96), dict(D=0), dict(qr=255), dict(kr=127), dict(vr=127), dict(orow=255),
                dict(qr=(1 << 22) + 8), dict(kr=(1 << 22) + 8), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
                dict(scale=math.inf), dict(scale=3e38), dict(cap=-1.0), dict(cap=math.inf), dict(cap=3e38), dict(cap=1e-44),
                dict(window=-1), dict(out=F, k=F, q=P(0x3000)), dict(out=P(0x2000)), dict(q=P(0x9000), orow=264)):
        assert status(**bad) == 1, bad
    for bad in (dict(q=MIS), dict(k=MIS), dict(v=MIS), dict(out=MIS), dict(qr=260), dict(lse=P(0x1001)), dict(starts=P(0x1001))):
        assert status(**bad) == 2, bad


def _pool(**kw):
    c = dict(table=0x1000, table_stride=4, refs=0x2000, seqs=3, max_pages=4, num_pages=8, page_size=16)
    c.update(kw)
    return pld._Pool(*[c[f] for f, _ in pld._Pool._fields_])


BAD_POOLS = [(dict(table=None), 1), (dict(refs=None), 1), (dict(seqs=0), 1), (dict(seqs=(1 << 20) + 1), 1), (dict(max_pages=0), 1),
             (dict(max_pages=5), 1), (dict(num_pages=0), 1), (dict(num_pages=(1 << 24) + 1), 1), (dict(page_size=8), 1),
             (dict(page_size=24), 1), (dict(page_size=8192), 1), (dict(max_pages=1 << 27, table_stride=1 << 27), 1),
             (dict(table=0x1002), 2), (dict(refs=0x2004), 2)]
I = P(0x4000)
WS = P(0x8000)


@no_gpu
def test_page_refusals():
    lib = pld._load()
    big = 1 << 30

    def layers(n=1, **kw):
        return (pld._Cache * n)(*[_cache(**kw) for _ in range(n)])

    take = dict(seq=I, need=I, count=2, status=I, ws=WS, wsb=big, stream=NULL)
    free = dict(seq=I, keep=I, count=2, stream=NULL)
    fork = dict(layers=layers(), n=1, src=I, dst=I, lens=I, count=2, status=I, ws=WS, wsb=big, stream=NULL)
    comp = dict(layers=layers(), n=1, map=I, used=I, table=I, ts=4, refs=I, ws=WS, wsb=big, stream=NULL)
    calls = ((lib.pld_pages_take, take), (lib.pld_pages_free, free), (lib.pld_pages_fork, fork), (lib.pld_pages_compact, comp))
    for fn, args in calls:
        assert fn(None, *args.values()) == 1
        for kw, want in BAD_POOLS:
            assert fn(_pool(**kw), *args.values()) == want, kw

    def status(fn, args, **kw):
        return fn(_pool(), *{**args, **kw}.values())

    for fn, args in calls[:3]:
        for bad in (dict(count=0), dict(count=4097)):
            assert status(fn, args, **bad) == 1
    for fn, args, names in ((lib.pld_pages_take, take, ("seq", "need", "status")), (lib.pld_pages_free, free, ("seq",)),
                            (lib.pld_pages_fork, fork, ("src", "dst", "lens", "status")),
                            (lib.pld_pages_compact, comp, ("map", "used", "table", "refs"))):
        for name in names:
            assert status(fn, args, **{name: NULL}) == 1, name
            assert status(fn, args, **{name: P(0x4002)}) == 2, name
    for fn, args in calls[:1] + calls[2:]:
        count = args.get("count", 1)
        need = lib.pld_pages_workspace_bytes(_pool(), count)
        assert need > 0
        for bad in (dict(ws=NULL), dict(ws=MIS), dict(wsb=need - 1)):
            assert status(fn, args, **bad) == 3, bad
    for fn, args in calls[2:]:
        for bad in (dict(layers=None), dict(n=-1), dict(n=65), dict(layers=layers(num_pages=9)),
                    dict(layers=layers(page_size=32, page_stride=32 * 2 * 64))):
            assert status(fn, args, **bad) == 1, bad
        for kw, want in BAD_CACHES:
            if "table" not in kw and "max_pages" not in kw and "num_pages" not in kw:
                assert status(fn, args, layers=layers(**kw)) == want, kw
        two = layers(2)
        two[1].slot_stride = 256
        assert status(fn, args, layers=two, n=2) == 1
    for bad in (dict(ts=3), dict(table=P(0x1000), ts=5)):
        assert status(lib.pld_pages_compact, comp, **bad) == 1, bad
    copy = dict(f=layers(), t=layers(), n=1, src=I, dst=I, slots=I, count=2, stream=NULL)
    for bad in (dict(f=None), dict(t=None), dict(n=0), dict(n=65), dict(src=NULL), dict(dst=NULL), dict(count=0),
                dict(count=(1 << 24) + 1), dict(t=layers(heads=1)), dict(t=layers(page_size=32, page_stride=32 * 2 * 64)),
                dict(t=layers(**Q8)), dict(t=layers(head_dim=128, slot_stride=256, head_stride=128, page_stride=16 * 256))):
        assert lib.pld_pages_copy(*{**copy, **bad}.values()) == 1, bad
    assert lib.pld_pages_copy(*{**copy, "slots": P(0x4001)}.values()) == 2


def test_workspace_bytes():
    lib = pld._load()
    for kw, want in BAD_POOLS:
        if want == 1:
            assert lib.pld_pages_workspace_bytes(_pool(**kw), 1) == 0
    for count in (0, -1, 4097):
        assert lib.pld_pages_workspace_bytes(_pool(), count) == 0
    assert lib.pld_pages_workspace_bytes(None, 1) == 0
    a, b = (lib.pld_pages_workspace_bytes(_pool(num_pages=n), 7) for n in (100, 1 << 24))
    assert 0 < a < b < 1 << 28


def test_host_tensors_and_odd_arguments_are_refused():
    t = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    k = torch.zeros(1, 16, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: pld.pld_prompt_attn(t, t, t, i, t), lambda: pld.pld_cache_write_packed(t, t, t, k, k, i[None], i, i, t),
                 lambda: pld.PageTable(i[None], i, 16),
                 lambda: PagePool([k], [k]), lambda: pld.PageLayers([k], [k, k]), lambda: pld.PageLayers([k], [k], [i], None)):
        with pytest.raises(TypeError):
            call()


def test_pools_that_are_not_whole():
    t, r, k = torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 16, 1, 64, dtype=torch.bfloat16)
    for args in (([], [], None, None, t, r), ([k], [k], None, None, t, None), ([k], [k], None, None, None, r)):
        with pytest.raises(TypeError):
            PagePool(*args)


def test_prepared_page_calls_keep_their_structs():
    """A prepared page call holds its pool and its array of caches by itself."""
    import gc
    pool = pld._Pool(0x7700, 8, 0x7800, 4, 8, 9, 16)
    layers = (pld._Cache * 2)(_cache(k=0x7770), _cache(k=0x7780))
    calls = [pld.Prepared("pld_pages_fork", (pool, layers, 2, 1, 1, 1, 1, 1, 1, 1, 0)),
             pld.Prepared("pld_pages_compact", (pool, layers, 2, 1, 1, 1, 8, 1, 1, 1, 0)),
             pld.Prepared("pld_pages_copy", (layers, layers, 2, 1, 1, 1, 1, 0)),
             pld.Prepared("pld_pages_take", (pool, 1, 1, 1, 1, 1, 1, 0)),
             pld.Prepared("pld_pages_free", (pool, 1, 1, 1, 0))]
    del pool, layers
    gc.collect()
    [_cache(k=i) for i in range(1000)]
    for c in calls:
        if c.name != "pld_pages_copy":
            assert c.args[0].contents.table == 0x7700 and c.args[0].contents.page_size == 16
    for a in (calls[0].args[1], calls[1].args[1], calls[2].args[0], calls[2].args[1]):
        assert [a[i].k for i in range(2)] == [0x7770, 0x7780]


@pytest.fixture
def on_host(monkeypatch):
    """The bindings with host tensors: what they hand to the library, whose host checks come before any launch."""
    monkeypatch.setattr(pld, "_need", lambda t, dtype, name, dims: t.stride())
    monkeypatch.setattr(pld, "_on_one_device", lambda *a: None)
    monkeypatch.setattr(pld, "_stream", lambda stream: 0)


def _host_pool(seqs=3, per=4, pages=9):
    """A PageTable, and no layers, of host tensors."""
    table, refs = torch.full((seqs, per), -1, dtype=torch.int32), torch.zeros(pages + 4, dtype=torch.int32)
    refs = refs[-refs.data_ptr() % 16 // 4:][:pages]
    return pld.PageTable(table, refs, 16)


@no_gpu
@pytest.mark.parametrize("seqs", [1, 3])
def test_compact_takes_the_stride_of_its_table(on_host, seqs):
    """A new table whose rows overlap is refused, as its size is not what the kernels would write."""
    p = _host_pool(seqs)
    ints = lambda n: torch.zeros(n, dtype=torch.int32)
    layers, ws = pld.PageLayers([], []), torch.zeros(1 << 16, dtype=torch.uint8)

    def call(table_out):
        return pld.pld_pages_compact(p, layers, ints(9), ints(1), ws, table_out=table_out, prepare=True)

    assert call(ints(64)[:seqs * 12].view(seqs, 12)[:, :4]).args[6].value == 12
    overlapping = [ints(4).expand(seqs, 4), ints(64).as_strided((seqs, 4), (3, 1))]
    for t in overlapping:
        c = call(t)
        assert c.args[6].value == (4 if seqs == 1 else t.stride(0))
        if seqs > 1:
            with pytest.raises(pld.PLDError) as e:
                c()
            assert e.value.status == 1


def test_a_refused_reservation_leaves_the_pool_as_it_was(on_host, monkeypatch):
    """More sequences than a call takes: refused, and calls of fewer keep their workspace."""
    monkeypatch.setattr(cache, "PageLayers", lambda *a: pld.PageLayers([], []))
    k = torch.zeros(9, 16, 1, 64, dtype=torch.bfloat16)
    pages = _host_pool()
    pool = PagePool([k], [k], table=pages.table, refs=pages.refs)
    for before in (0, 3):
        if before:
            pool.reserve(before)
        kept, most = pool.workspace, pool.most
        i = torch.zeros(pld.PLD_MAX_PAGE_ENTRIES + 1, dtype=torch.int32)
        for call in (lambda: pool.reserve(len(i)), lambda: pool.take(i, i, i), lambda: pool.fork(i, i, i, i)):
            with pytest.raises(pld.PLDError):
                call()
            assert pool.workspace is kept and pool.most == most and pool.grown == []
    pool.reserve(2)
    assert pool.workspace is kept
    pool.reserve(pld.PLD_MAX_PAGE_ENTRIES)
    assert pool.grown == [kept] and pool.workspace.numel() == pld.pld_pages_workspace_bytes(pool.pages, pld.PLD_MAX_PAGE_ENTRIES)


def test_a_refused_pool_leaves_its_caches_as_they_were():
    caches = [cache.PagedCache(2, 40, 1, 64, page_size=16, device="cpu") for _ in range(2)]     # (host tensors are refused)
    tables = [c.table for c in caches]
    with pytest.raises(TypeError):
        PagePool.of_caches(caches, seqs=3)
    assert all(c.table is t for c, t in zip(caches, tables))


def test_a_pool_that_only_copies_says_so(on_host, monkeypatch):
    """Without a table and references: calls that need them are refused with the reason."""
    monkeypatch.setattr(cache, "PageLayers", lambda *a: pld.PageLayers([], []))
    i = torch.zeros(2, dtype=torch.int32)
    pool = PagePool([i], [i])
    for call in (lambda: pool.take(i, i, i), lambda: pool.free(i), lambda: pool.fork(i, i, i, i), lambda: pool.compact(i, i),
                 lambda: pool.reserve(3)):
        with pytest.raises(TypeError, match="only copies"):
            call()
    assert pool.workspace is None and pool.most == 0


def test_scales_of_some_layers_alone_are_refused():
    k = torch.zeros(1, 16, 1, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="scales"):
        pld.PageLayers([k, k], [k, k], [k[..., 0], None], [k[..., 0], None])
