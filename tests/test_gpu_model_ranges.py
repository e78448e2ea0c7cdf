"""The model-side calls at the ends of the ranges that their arguments are documented for.
References are plain, in 64 bits; bounds come from the arithmetic (see model_ref.py).
"""
import pytest
import torch

import paper_2412_01447_amd as pld
from gpu_helpers import dev, say
from model_ref import U

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
