"""Host checks of the model-side calls at the ends of their documented ranges (CPU only)."""
import gc
import weakref

import paper_2412_01447_amd as pld
from paper_2412_01447_amd.cache import PagedCache
from paper_2412_01447_amd.step import DraftStep
from test_model_abi import ATTN, ROWS, _cache, no_gpu


@no_gpu
def test_largest_cap():
    """Twice the cap in log2 units is fp32: a cap of 2^126 is in range (the next check speaks),
    one of 1.5e38 is not."""
    lib = pld._load()
    for fn, args in ((lib.pld_cache_attn, ATTN), (lib.pld_cache_attn_rows, ROWS)):
        assert fn(_cache(), *{**args, "cap": 1.5e38}.values()) == 1
    assert lib.pld_cache_attn(_cache(), *{**ATTN, "cap": 2.0 ** 126, "wsb": 0}.values()) == 3


def test_workspace_of_the_most_rows_serves_fewer():
    """The attention's workspace never falls as the rows of a sequence grow (the rows are split
    into even groups, so that more rows can have smaller ones)."""
    for D in (64, 128, 256):
        for Hq, heads in ((1, 1), (8, 8), (8, 1), (40, 8), (12, 4), (56, 8), (16, 1), (96, 2), (4096, 1)):
            sizes = [pld.pld_cache_attn_workspace_bytes(3, n, Hq, heads, D) for n in [*range(1, 400), 1000, 5000, 65535]]
            assert sizes[0] > 0 and sizes == sorted(sizes), (D, Hq, heads)
    cache = PagedCache(2, 100, 1, 64, page_size=16, device="cpu")
    cache.reserve(22, 8)
    ws = cache.workspace
    for n in range(1, 22):
        cache.reserve(n, 8)
    assert cache.workspace is ws


def test_buffers_that_plans_point_to_are_kept():
    """set_logprobs() replaces buffers; those that plans and graphs made before write to stay
    allocated as long as the step does."""
    step = DraftStep(2, 100, 4, device="cpu")
    old = []
    for top in (3, 0, 5):
        step.set_logprobs(50, bf16=True, top=top)
        old += [weakref.ref(t) for t in (step.logprob, step.logprob_entropy, step.logprob_ws, step.top_ids, step.top_logprobs)
                if t is not None]
    step.set_logprobs(None, bf16=True)
    step.set_logprobs(20, bf16=True)
    gc.collect()
    assert len(old) == 13 and all(ref() is not None for ref in old)


def test_buffers_that_sampling_replaces_are_kept():
    """set_sampling() too."""
    step = DraftStep(2, 100, 4, device="cpu")
    old = [weakref.ref(step.workspace)]
    for V in (1000, 200000):
        step.set_sampling(0.7, V, bf16=False)
        old += [weakref.ref(t) for t in (step.workspace, step.uniforms, step.row_sample)]
    step.set_sampling(None, 0, False)
    step.set_sampling(0.7, 1000, bf16=False)
    gc.collect()
    assert all(ref() is not None for ref in old)
