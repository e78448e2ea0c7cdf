"""Host checks of the model-side calls at the ends of their documented ranges (CPU only)."""
import paper_2412_01447_amd as pld
from test_model_abi import ATTN, ROWS, _cache, no_gpu


@no_gpu
def test_largest_cap():
    """Twice the cap in log2 units is fp32: a cap of 2^126 is in range (the next check speaks),
    one of 1.5e38 is not."""
    lib = pld._load()
    for fn, args in ((lib.pld_cache_attn, ATTN), (lib.pld_cache_attn_rows, ROWS)):
        assert fn(_cache(), *{**args, "cap": 1.5e38}.values()) == 1
    assert lib.pld_cache_attn(_cache(), *{**ATTN, "cap": 2.0 ** 126, "wsb": 0}.values()) == 3
