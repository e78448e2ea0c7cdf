"""include/pld_model.h and its calls' host checks (CPU only; no kernel is launched here)."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

import paper_2412_01447_amd as pld
from paper_2412_01447_amd.cache import PagedCache
from paper_2412_01447_amd.step import DraftStep

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "pld_model.h")
P = ctypes.c_void_p
F = P(0x1000)            # placeholder pointers, never dereferenced (the host check fails first)
MIS = P(0x1004)
NULL = None
no_gpu = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="placeholder pointers are only used where no GPU is visible")


def _declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(pld_\w+)\s*\(", text)))


def test_declared_calls_are_exported_and_bound():
    assert _declared() == ["pld_cache_attn", "pld_cache_attn_rows", "pld_cache_attn_workspace_bytes",
                           "pld_cache_write", "pld_model_version", "pld_token_logprobs",
                           "pld_token_logprobs_workspace_bytes"]
    for n in _declared():
        assert hasattr(pld._load(), n) and hasattr(pld, n)
        assert len(getattr(pld._load(), n).argtypes) == len(pld._SIGNATURES[n][0])
    m = re.search(r"#define PLD_MODEL_ABI_VERSION (\d+)", open(HEADER).read())
    assert pld.pld_model_version() == int(m.group(1))
    m = re.search(r"#define PLD_MAX_TOP (\d+)", open(HEADER).read())
    assert pld.PLD_MAX_TOP == int(m.group(1))


def test_argument_counts_and_the_struct_match_the_header(tmp_path):
    """Every call with the header's number of arguments; the struct's offsets as C has them."""
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    for n in _declared():
        args = re.search(r"\b%s\s*\(([^)]*)\)" % n, text).group(1).strip()
        assert len(pld._SIGNATURES[n][0]) == (0 if args == "void" else args.count(",") + 1), n
    fields = [f for f, _ in pld._Cache._fields_]
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include "pld_model.h"\nint main(void) {\n' + "".join(
        f'printf("%zu\\n", offsetof(pld_cache, {f}));\n' for f in fields) + 'printf("%zu\\n", sizeof(pld_cache));\nreturn 0; }\n')
    for cc, std in (("gcc", "-std=c99"), ("g++", "-std=c++17")):
        subprocess.run([cc, std, "-Wall", "-Wextra", "-pedantic", "-Werror", "-x", "c" if cc == "gcc" else "c++",
                        "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "t")], check=True)
        out = subprocess.run([str(tmp_path / "t")], check=True, capture_output=True, text=True).stdout.split()
        assert [int(x) for x in out] == [getattr(pld._Cache, f).offset for f in fields] + [ctypes.sizeof(pld._Cache)]


def _cache(**kw):
    c = dict(k=0x1000, v=0x2000, dtype=pld.PLD_BF16, k_scale=None, v_scale=None, scale_page_stride=0,
             page_stride=16 * 2 * 64, slot_stride=128, head_stride=64, table=0x3000, table_stride=4,
             num_pages=8, page_size=16, max_pages=4, heads=2, head_dim=64)
    c.update(kw)
    return pld._Cache(*[c[f] for f, _ in pld._Cache._fields_])


Q8 = dict(dtype=pld.PLD_E4M3, k_scale=0x4000, v_scale=0x5000, scale_page_stride=32)
BAD_CACHES = [(dict(k=None), 1), (dict(v=None), 1), (dict(table=None), 1), (dict(dtype=0), 1), (dict(dtype=3), 1),
              (dict(k_scale=0x4000), 1), (dict(Q8, k_scale=None), 1), (dict(Q8, v_scale=None), 1),
              (dict(Q8, scale_page_stride=31), 1), (dict(Q8, scale_page_stride=34), 2), (dict(Q8, k_scale=0x4004), 2),
              (dict(page_size=8), 1), (dict(page_size=24), 1), (dict(page_size=8192), 1), (dict(num_pages=0), 1),
              (dict(max_pages=0), 1), (dict(max_pages=5), 1), (dict(max_pages=1 << 27, table_stride=1 << 27), 1),
              (dict(heads=0), 1), (dict(heads=1025), 1), (dict(head_dim=96), 1), (dict(head_dim=0), 1),
              (dict(slot_stride=63), 1), (dict(head_stride=32), 1), (dict(page_stride=0), 1), (dict(k=0x1008), 2),
              (dict(v=0x2008), 2), (dict(page_stride=2052), 2), (dict(slot_stride=132), 2), (dict(head_stride=68), 2),
              (dict(table=0x3002), 2), (dict(Q8, slot_stride=136), 2)]

WRITE = dict(q=F, qs=512, qr=256, k=F, ks=256, kr=128, v=F, vs=256, vr=128, qn=NULL, kn=NULL, eps=1e-6, rope=F, rs=64,
             n_pos=9, rot=64, pairs=0, lens=F, dl=NULL, B=2, n=2, Hq=4, out=F, os=512, orow=256, stream=NULL)
ATTN = dict(q=F, qs=512, qr=256, lens=F, dl=NULL, B=2, n=2, Hq=4, scale=1.0, cap=0.0, window=0, out=F, os=512, orow=256,
            lse=F, ws=F, wsb=1 << 30, stream=NULL)
ROWS = dict(q=F, qs=512, qr=256, lens=F, row=F, heads=F, R=3, lse=F, B=2, n=2, Hq=4, scale=1.0, cap=0.0, window=0, attn=F,
            as_=300, ar=100, keys=100, stream=NULL)
LP = dict(z=F, dtype=0, ls=200, lr=100, V=100, n=2, tok=F, cnt=NULL, B=2, tau=1.0, lp=F, ent=NULL, top=3, ids=F, tlp=F,
          ws=F, wsb=1 << 30, stream=NULL)


@no_gpu
@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_bad_caches(kw, status):
    """A v that is missing or misaligned does not matter to the rows call."""
    lib = pld._load()
    for fn, args in ((lib.pld_cache_write, WRITE), (lib.pld_cache_attn, ATTN), (lib.pld_cache_attn_rows, ROWS)):
        args = dict(args)
        if fn is lib.pld_cache_attn_rows and ("v" in kw or kw.get("v_scale", 1) is None):
            args["R"] = 0                    # so that nothing is launched
            assert fn(_cache(**kw), *args.values()) == 1
        else:
            assert fn(_cache(**kw), *args.values()) == status


@no_gpu
def test_host_checks():
    lib = pld._load()

    def refused(fn, base, status, *first, **kw):
        for name, value in kw.items():
            assert fn(*first, *{**base, name: value}.values()) == status, (name, value)

    c = _cache()
    w = lib.pld_cache_write
    assert w(None, *WRITE.values()) == 1
    for name in ("q", "k", "v", "lens", "out"):
        refused(w, WRITE, 1, c, **{name: NULL})
    for bad in (dict(B=0), dict(B=65536), dict(n=0), dict(n=65536), dict(Hq=3), dict(Hq=0), dict(Hq=4098), dict(qr=255),
                dict(qs=255), dict(kr=127), dict(vs=100), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf),
                dict(pairs=2), dict(n_pos=0), dict(rot=12), dict(rot=72), dict(rot=0), dict(rs=60)):
        refused(w, WRITE, 1, c, **bad)
    for bad in (dict(q=MIS), dict(k=MIS), dict(v=MIS), dict(out=MIS), dict(qr=260), dict(ks=260), dict(qn=MIS), dict(kn=MIS),
                dict(rope=MIS), dict(rs=66)):
        refused(w, WRITE, 2, c, **bad)
    a = lib.pld_cache_attn
    for name in ("q", "lens", "out"):
        refused(a, ATTN, 1, c, **{name: NULL})
    for bad in (dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(cap=-1.0), dict(cap=math.inf), dict(window=-1),
                dict(os=255), dict(B=0), dict(n=0), dict(Hq=5)):
        refused(a, ATTN, 1, c, **bad)
    refused(a, ATTN, 2, c, out=MIS)
    refused(a, ATTN, 2, c, lse=P(0x1001))
    need = pld.pld_cache_attn_workspace_bytes(2, 2, 4, 2, 64)
    refused(a, ATTN, 3, c, ws=NULL)
    refused(a, ATTN, 3, c, ws=MIS)
    refused(a, ATTN, 3, c, wsb=need - 1)
    r = lib.pld_cache_attn_rows
    for name in ("q", "lens", "row", "heads", "lse", "attn"):
        refused(r, ROWS, 1, c, **{name: NULL})
    for bad in (dict(R=0), dict(R=65536), dict(keys=0), dict(as_=99), dict(ar=99), dict(scale=0.0), dict(window=-1)):
        refused(r, ROWS, 1, c, **bad)
    refused(r, ROWS, 2, c, attn=P(0x1002))
    lp = lib.pld_token_logprobs
    for name in ("z", "tok", "lp", "ids", "tlp"):
        refused(lp, LP, 1, **{name: NULL})
    for bad in (dict(dtype=2), dict(V=0), dict(n=0), dict(n=65536), dict(B=0), dict(B=65536), dict(top=-1), dict(top=65),
                dict(lr=99), dict(ls=99), dict(tau=0.0), dict(tau=math.inf), dict(tau=math.nan), dict(tau=1e-300)):
        refused(lp, LP, 1, **bad)
    refused(lp, LP, 2, z=P(0x1002))
    refused(lp, LP, 3, ws=NULL)
    refused(lp, LP, 3, ws=MIS)
    refused(lp, LP, 3, wsb=pld.pld_token_logprobs_workspace_bytes(2, 2, 100, 0, 3) - 1)


@no_gpu
def test_limits():
    """The largest strides and lengths that the kernels' 32-bit offsets are made for, and one
    call whose outputs would be read while they are written."""
    lib = pld._load()
    calls = ((lib.pld_cache_write, WRITE), (lib.pld_cache_attn, ATTN), (lib.pld_cache_attn_rows, ROWS))
    for kw in (dict(slot_stride=(1 << 24) + 8), dict(page_stride=(1 << 34) + 8),
               dict(Q8, scale_page_stride=(1 << 31) + 4)):
        for fn, args in calls:
            assert fn(_cache(**kw), *args.values()) == 1, kw
    # in range: the next check speaks
    for kw in (dict(slot_stride=1 << 24, k=0x1008), dict(page_stride=1 << 34, k=0x1008),
               dict(Q8, scale_page_stride=1 << 31, k_scale=0x4004)):
        for fn, args in calls:
            assert fn(_cache(**kw), *args.values()) == 2, kw
    n_keys = 2 ** 31 - 65536
    assert lib.pld_cache_attn_rows(_cache(), *{**ROWS, "keys": n_keys, "as_": 3 * n_keys, "ar": n_keys}.values()) == 1
    for bad in (dict(scale=3e38), dict(cap=3e38), dict(cap=1e-44)):
        for fn, args in calls[1:]:
            assert fn(_cache(), *{**args, **bad}.values()) == 1, bad
    same = P(0x8000)
    assert lib.pld_cache_attn(_cache(), *{**ATTN, "q": same, "out": same}.values()) == 1
    for other in (dict(os=520), dict(orow=264, os=600)):
        assert lib.pld_cache_write(_cache(), *{**WRITE, "q": same, "out": same, **other}.values()) == 1


def test_workspace_bytes():
    for args in ((0, 1, 8, 2, 64), (65536, 1, 8, 2, 64), (1, 0, 8, 2, 64), (1, 1, 8, 3, 64), (1, 1, 8, 2, 96), (1, 1, 0, 2, 64)):
        assert pld.pld_cache_attn_workspace_bytes(*args) == 0
    for args in ((0, 1, 5, 0, 1), (1, 65536, 5, 0, 1), (1, 1, 0, 0, 1), (1, 1, 5, 2, 1), (1, 1, 5, 0, 65), (1, 1, 5, 0, -1)):
        assert pld.pld_token_logprobs_workspace_bytes(*args) == 0
    assert pld.pld_cache_attn_workspace_bytes(64, 17, 64, 8, 128) > 0
    assert pld.pld_token_logprobs_workspace_bytes(65535, 65535, 2 ** 31 - 1, 1, 64) > 0


def test_prepared_call_keeps_the_struct():
    """A prepared call holds its struct by itself."""
    import gc
    call = pld.Prepared("pld_cache_attn", (_cache(k=0x7770),) + tuple(
        getattr(v, "value", v) for v in ATTN.values()))
    gc.collect()
    [_cache(k=i) for i in range(1000)]
    assert call.args[0].contents.k == 0x7770 and call.args[0].contents.head_dim == 64


def test_host_tensors_are_refused():
    t = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16)
    k = torch.zeros(1, 16, 1, 64, dtype=torch.bfloat16)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        pld.pld_cache_attn(t, k, k, i[None], i, t, i)
    with pytest.raises(TypeError):
        pld.pld_cache_write(t, k, k, k, k, i[None], i, t)
    with pytest.raises(TypeError):
        pld.pld_cache_attn_rows(t, k, i[None], i, i, i, i.float(), i.float())
    with pytest.raises(TypeError):
        pld.pld_token_logprobs(torch.zeros(1, 1, 5), i[None], torch.zeros(1, 1), i)


def test_step_buffers_of_log_probabilities():
    s = DraftStep(2, 100, 4, device="cpu")
    assert s.logprob is None
    s.set_logprobs(50, bf16=True, top=3, temperature=0.5)
    assert s.logprob.shape == (2, 5) and s.top_ids.shape == (2, 5, 3) and s.logprob_temperature == 0.5
    with pytest.raises(ValueError):
        s.set_logprobs(50, bf16=True, top=65)
    s.set_logprobs(50, bf16=False)
    assert s.top_ids is None
    s.set_logprobs(None, bf16=False)
    assert s.logprob is None


def test_cache_layouts():
    """Rows of less than a 128-byte line lie slot by slot within a head, others head by head."""
    a = PagedCache(2, 40, 3, 64, page_size=16, device="cpu")
    assert a.k.shape == a.v.shape == (6, 16, 3, 64) and a.k.stride() == a.v.stride() == (16 * 3 * 64, 3 * 64, 64, 1)
    b = PagedCache(2, 40, 3, 64, page_size=16, dtype=torch.float8_e4m3fn, device="cpu", num_pages=9)
    assert b.k.shape == (9, 16, 3, 64) and b.k.stride() == b.v.stride() == (16 * 3 * 64, 64, 16 * 64, 1)
    assert b.k_scale.shape == (9, 3, 16) and b.table.shape == (2, 3)
    with pytest.raises(TypeError):
        PagedCache(2, 40, 3, 64, dtype=torch.float16, device="cpu")
