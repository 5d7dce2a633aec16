"""Edges of the paged-cache operators: what their weights add up to, NaN, infinities, lengths past the table, indexes that are
none, calls that the documentation allows and few programs make."""
import numpy as np
import pytest
import torch

from oracle import paged_kv as O
from tests.test_gpu_paged_kv import EPS, LAYOUTS, Cache, _check_attention, _check_score, _queries

pytestmark = pytest.mark.gpu

TINY, B128, B64, F128, B32, B96 = LAYOUTS[0], LAYOUTS[1], LAYOUTS[3], LAYOUTS[4], LAYOUTS[8], LAYOUTS[9]
ids = lambda x: "-".join(map(str, x))   # noqa: E731


def _attend(c, q, cu, most, Hq, window=0, sinks=0, use_ws=False, must_split=None):
    """(out, lse) of a call, with a workspace if asked for; must_split: whether the call has to need one."""
    from paper_2601_19404_amd import binding as rpo
    need = rpo.rpo_attn_paged_ws_bytes(c.dev, q.shape[0], most, max(c.lens), Hq, window, sinks)
    if must_split is not None:
        assert (need > 0) == must_split
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need and use_ws else None
    out, lse = torch.full_like(q.contiguous(), 7.0), torch.full((q.shape[0], Hq), 7.0, device="cuda")
    rpo.rpo_attn_paged(c.dev, q, cu, most, out, window, sinks, None, lse, ws, max(c.lens))
    torch.cuda.synchronize()
    return out, lse


def _rewrite(c, s, slots, k=None, v=None):
    """Other keys or values (broadcast to [slots, KV heads, channels]) in slots of a sequence."""
    at = torch.as_tensor(slots)
    for own, x in ((c.k[s], k), (c.v[s], v)):
        if x is not None:
            own[at] = torch.as_tensor(x).to(own.dtype).expand(len(at), c.Hkv, c.dh)
    pool = c.pool.cpu()
    c.write(pool, s, at, c.k[s][at], c.v[s][at])
    c.pool.copy_(pool)


# Weights that are divided by their own sum leave a value that all tokens share as it is: sums of T terms in fp32 are off by
# less than T 2^-24 < 2^-12 of it, and half a step of bf16 is at least 2^-9 of a value, so bf16 results are equal; fp32 ones
# are off by T roundings in each of the two sums, one in the product, one in the quotient.
@pytest.mark.parametrize("layout", [TINY, B128, B64, B32, F128, B96], ids=ids)
@pytest.mark.parametrize("new", [40, 150])
@pytest.mark.parametrize("use_ws", [False, True])
def test_chunks_over_equal_values_return_the_value(layout, new, use_ws):
    Hq, Hkv, dh, dtype, pt = layout
    lens, news = [1500, 700, new], [new, 33, new]
    c = Cache(lens, Hkv, dh, pt, dtype, seed=dh)
    value = torch.randn(Hkv, dh, generator=torch.Generator().manual_seed(1)).to(c.k[0].dtype)
    for s, n in enumerate(lens):
        _rewrite(c, s, range(n), v=value)
    q, cu, _ = _queries(news, Hq, dh, dtype, seed=dh)
    want = value.repeat_interleave(Hq // Hkv, dim=0).view(1, -1).expand(q.shape[0], -1)
    for window, sinks in ((0, 0), (1, 0), (200, 3)):
        out, _ = _attend(c, q, cu, max(news), Hq, window, sinks, use_ws)
        if dtype == "bf16":
            assert torch.equal(out.cpu(), want), (window, sinks)
        else:
            off = (out.cpu() - want).abs() - (2 * max(lens) + 4) * EPS * want.abs()
            assert off.max() <= 0, (window, sinks, off.max())
