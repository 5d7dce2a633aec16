"""Edges of the paged-cache operators: what their weights add up to, NaN, infinities, lengths past the table, indexes that are
none, calls that the documentation allows and few programs make."""
import numpy as np
import pytest
import torch

from oracle import paged_kv as O
from tests.test_gpu_paged_kv import EPS, LAYOUTS, Cache, _queries, _tolerance

pytestmark = pytest.mark.gpu

TINY, B128, B64, F128, B32, B96 = LAYOUTS[0], LAYOUTS[1], LAYOUTS[3], LAYOUTS[4], LAYOUTS[8], LAYOUTS[9]
ids = lambda x: "-".join(map(str, x))   # noqa: E731


def _chunk_tolerance(T, dh, ref, mag, big, dtype):
    """The bound of a chunk, whose bf16 weights are rounded in the products and in the sum that divides them.  With w_j (1 + d_j),
    |d_j| <= 2^-8, in both, the quotient is off by sum p_j d_j (v_j - out) to first order, at most 2^-8 (sum p_j |v_j| + |out|):
    2^-8 |out| more than with the exact sum, the second order within the factor 1 + 2^-7 as in _tolerance."""
    more = 0.0 if dtype == "f32" else 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -7)
    return _tolerance(T, dh, ref, mag, big, dtype) + more


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


@pytest.mark.parametrize("layout", [B128, B64, B32, (32, 2, 128, "bf16", 256), (24, 3, 64, "bf16", 128)], ids=ids)
@pytest.mark.parametrize("window,sinks", [(1, 1), (1, 4), (2, 0), (3, 2), (12, 0)])
def test_chunks_over_a_few_visible_tokens_stay_within_their_roundings(layout, window, sinks):
    """Where a few weights make the whole sum, their roundings do not even out."""
    Hq, Hkv, dh, dtype, pt = layout
    lens, news = [300, 160, 40], [150, 44, 40]
    c = Cache(lens, Hkv, dh, pt, dtype, seed=window + sinks)
    q, cu, at = _queries(news, Hq, dh, dtype, seed=7 * window + sinks)
    out, _ = _attend(c, q, cu, max(news), Hq, window, sinks)
    for s, (T, n) in enumerate(zip(lens, news)):
        rows = q[at[s]: at[s + 1]].float().cpu().numpy().reshape(n, Hq, dh)
        ref, _, _, mag, big = O.attention(rows, c.k[s].float().numpy(), c.v[s].float().numpy(), dh ** -0.5, window, sinks)
        off = np.abs(out[at[s]: at[s + 1]].float().cpu().numpy().reshape(ref.shape) - ref)
        assert (off - _chunk_tolerance(T, dh, ref, mag, big, dtype)).max() <= 0, s


# new 1: the kernel for few rows, 40: the one for chunks; both are split over the tokens if there is a workspace
@pytest.mark.parametrize("layout", [TINY, B128, B64, F128], ids=ids)
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("use_ws", [False, True])
def test_a_nan_in_a_query_head_is_seen_in_it_alone(layout, new, use_ws):
    Hq, Hkv, dh, dtype, pt = layout
    c = Cache([2176, 257], Hkv, dh, pt, dtype, seed=2)
    q, cu, _ = _queries([new, new], Hq, dh, dtype, seed=3)
    q = q.clone()
    want, want_lse = _attend(c, q, cu, new, Hq, use_ws=use_ws, must_split=True)
    row, head = 2 * new - 1, Hq - 1
    q[row, head * dh + 1] = float("nan")
    out, lse = _attend(c, q, cu, new, Hq, use_ws=use_ws)
    assert out[row, head * dh:].isnan().all() and lse[row, head].isnan()
    out[row, head * dh:], lse[row, head] = want[row, head * dh:], want_lse[row, head]
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("layout", [TINY, B128, B64, F128], ids=ids)
@pytest.mark.parametrize("slot", [256, 255, 100, 0])
@pytest.mark.parametrize("use_ws", [False, True])
def test_a_nan_in_a_key_reaches_the_single_token_that_sees_it(layout, slot, use_ws):
    """Slot 256 of 257 is the only token of its piece: the newest one."""
    Hq, Hkv, dh, dtype, pt = layout
    c = Cache([2176, 257], Hkv, dh, pt, dtype, seed=2)
    q, cu, _ = _queries([1, 1], Hq, dh, dtype, seed=3)
    want, want_lse = _attend(c, q, cu, 1, Hq, use_ws=use_ws, must_split=True)
    bad = c.k[1][slot:slot + 1].clone()
    bad[:, Hkv - 1, dh - 1] = float("nan")
    _rewrite(c, 1, [slot], k=bad)
    out, lse = _attend(c, q, cu, 1, Hq, use_ws=use_ws)
    first = (Hkv - 1) * (Hq // Hkv)                    # of the heads that read the last KV head
    assert out[1, first * dh:].isnan().all() and lse[1, first:].isnan().all()
    assert torch.equal(out[0], want[0]) and torch.equal(lse[0], want_lse[0])
    assert torch.equal(out[1, : first * dh], want[1, : first * dh]) and torch.equal(lse[1, :first], want_lse[1, :first])


@pytest.mark.parametrize("layout", [TINY, B128, B96], ids=ids)
@pytest.mark.parametrize("over,news", [([1, 0, 3], [1, 1, 1]), ([5, 200, 2 ** 30], [9, 150, 20]),
                                       ([0, 2 ** 31 - 1 - 128, 40], [128, 1, 40])])
def test_append_drops_the_rows_behind_the_table(layout, over, news):
    """Lengths past what the table holds (128 slots): rows behind its end are dropped, the others land in their slots, and
    tokens that are there stay."""
    from paper_2601_19404_amd import binding as rpo
    _, Hkv, dh, dtype, pt = layout
    S, cap = 3, 128
    c = Cache([cap] * S, Hkv, dh, pt, dtype, seed=3, stale=5.0)
    lens = [cap + x for x in over]
    c.dev.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    rows = torch.randn(sum(news), 2, Hkv, dh, generator=torch.Generator().manual_seed(1)).to(c.pool.dtype)
    want, row = c.pool.cpu().clone(), 0
    for s in range(S):
        slots = torch.arange(lens[s] - news[s], lens[s])
        keep = (slots >= 0) & (slots < cap)
        c.write(want, s, slots[keep], rows[row: row + news[s]][keep, 0], rows[row: row + news[s]][keep, 1])
        row += news[s]
    cu = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32).cuda()
    flat = rows.cuda().view(sum(news), -1)
    rpo.rpo_kv_append(c.dev, flat[:, : Hkv * dh], flat[:, Hkv * dh:], cu, max(news))
    torch.cuda.synchronize()
    assert torch.equal(c.pool.cpu(), want)


def test_a_decode_loop_at_a_full_cache_leaves_it_alone():
    """Rows that find no room are dropped, and attention goes on over the tokens that are there."""
    from paper_2601_19404_amd import binding as rpo
    Hq, Hkv, dh, dtype, pt = B128
    c = Cache([128], Hkv, dh, pt, dtype, seed=3)
    before = c.pool.clone()
    q, cu, _ = _queries([1], Hq, dh, dtype, seed=3)
    want, want_lse = _attend(c, q, cu, 1, Hq)
    for step in range(1, 4):
        c.dev.lens.fill_(128 + step)
        rpo.rpo_kv_append(c.dev, q[:, :256], q[:, 256:512], cu, 1)
        out, lse = _attend(c, q, cu, 1, Hq)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert torch.equal(c.pool.view(torch.uint8), before.view(torch.uint8))


@pytest.mark.parametrize("layout", [TINY, B128, B64, F128, B96], ids=ids)
@pytest.mark.parametrize("new", [1, 8, 150])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 3)])
def test_rows_whose_lse_is_minus_infinity_give_no_score_whatever_their_queries_hold(layout, new, window, sinks):
    """Rows of a padded batch, say: lse -infinity, queries of NaN, infinities and numbers whose products overflow."""
    from paper_2601_19404_amd import binding as rpo
    Hq, Hkv, dh, dtype, pt = layout
    lens, news = [700, 160, 30], [new, new, min(new, 7)]
    c = Cache(lens, Hkv, dh, pt, dtype, seed=2)
    q, cu, _ = _queries(news, Hq, dh, dtype, seed=3)
    q, n = q.clone(), sum(news)
    _, lse = _attend(c, q, cu, new, Hq, window, sinks)
    dead = torch.zeros(n, Hq, dtype=torch.bool, device="cuda")
    dead[::3] = dead[n - 1] = True                     # whole rows, the last one among them
    dead[1::3, Hq - 1] = True                          # and single heads
    lse[dead] = -float("inf")
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device="cuda").to(q.dtype)
    bad = bad[torch.arange(n * Hq, device="cuda") % 4].view(n, Hq, 1)
    scores = []
    for x in (torch.zeros_like(bad), bad):
        rows = torch.where(dead[..., None], x, q.view(n, Hq, dh)).view(n, -1).contiguous()
        need = rpo.rpo_kv_score_ws_bytes(c.dev, n, new, 700, Hq, window, sinks)
        for use_ws in (False, True):
            ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need and use_ws else None
            score = torch.zeros(3, Hkv, 700, device="cuda")
            rpo.rpo_kv_score(c.dev, rows, cu, new, lse, None, score, window, sinks, ws_dev=ws, max_len=700)
            scores.append(score)
    torch.cuda.synchronize()
    assert all(bool(s.isfinite().all()) for s in scores)
    assert torch.equal(scores[0], scores[2]) and torch.equal(scores[1], scores[3])
    live = torch.where(dead, 0.0, 1.0).view(n, Hkv, -1).sum(dim=(0, 2)).tolist()
    for h in range(Hkv):                               # every live row and head gives its weights, which add up to 1
        assert abs(scores[3][:, h].double().sum().item() - live[h]) <= 1e-3 * live[h]


def test_binding_refuses_numbers_that_32_bits_do_not_hold():
    from paper_2601_19404_amd import binding as rpo
    Hq, Hkv, dh, dtype, pt = B128
    c = Cache([100], Hkv, dh, pt, dtype, seed=1)
    to = Cache([0], Hkv, dh, pt, dtype, seed=2, cap=64, stale=0.0)
    q, cu, _ = _queries([2], Hq, dh, dtype, seed=1)
    out, lse, score = torch.zeros_like(q), torch.zeros(2, Hq, device="cuda"), torch.zeros(1, Hkv, 100, device="cuda")
    kept, big = torch.zeros(100, dtype=torch.int32, device="cuda"), 2 ** 32
    before = c.pool.clone()
    for call in (lambda: rpo.rpo_attn_paged(c.dev, q, cu, 2, out, big), lambda: rpo.rpo_attn_paged(c.dev, q, cu, 2, out, 5, big),
                 lambda: rpo.rpo_attn_paged(c.dev, q, cu, big + 2, out), lambda: rpo.rpo_attn_paged(c.dev, q, cu, 2, out, max_len=big),
                 lambda: rpo.rpo_kv_score(c.dev, q, cu, 2, lse, None, score, big),
                 lambda: rpo.rpo_kv_score(c.dev, q, cu, big + 2, lse, None, score),
                 lambda: rpo.rpo_kv_append(c.dev, q[:, :256], q[:, :256], cu, big + 2),
                 lambda: rpo.rpo_kv_evict(c.dev, score, 50, big, 0, to.dev, to.dev.lens, kept),
                 lambda: rpo.rpo_kv_evict(c.dev, score, 50, 0, big, to.dev, to.dev.lens, kept),
                 lambda: rpo.rpo_kv_evict(c.dev, score, 50 - big, 0, 0, to.dev, to.dev.lens, kept)):
        with pytest.raises(ValueError):
            call()
    torch.cuda.synchronize()
    assert torch.all(out == 0) and torch.all(score == 0) and torch.equal(c.pool.view(torch.uint8), before.view(torch.uint8))


def test_binding_refuses_cache_sizes_below_one():
    from paper_2601_19404_amd import binding as rpo
    c = Cache([100], 2, 128, 64, "bf16", seed=1)
    for pt, heads, dh in ((64, 2, 0), (64, 2, -128), (0, 2, 128), (64, -2, 128), (64, 2, 2 ** 32 + 128)):
        with pytest.raises(ValueError):
            rpo.PagedKV(c.pool, c.dev.table, c.dev.lens, pt, heads, dh)


def test_a_pool_of_one_page_whose_stride_means_nothing():
    from paper_2601_19404_amd import binding as rpo
    Hq, Hkv, dh, dtype, pt = B128
    page = torch.zeros(2 * Hkv * pt * dh, dtype=torch.bfloat16, device="cuda")
    pool = page.as_strided((1, page.numel()), (1, 1))
    lens, table = torch.tensor([3], dtype=torch.int32).cuda(), torch.zeros(1, 1, dtype=torch.int32).cuda()
    kv = rpo.PagedKV(pool, table, lens, pt, Hkv, dh)
    q, cu, _ = _queries([3], Hq, dh, dtype, seed=1)
    rpo.rpo_kv_append(kv, q[:, :256], q[:, 256:512], cu, 3)
    torch.cuda.synchronize()
    assert torch.equal(page[: 3 * dh].view(3, dh), q[:, :dh])


BAD_CU = [[0, 40, 80], [-3, 1, 2], [6, 2, 1 << 30], [9, 9, 9], [0, 3, -5], [-(1 << 31), (1 << 31) - 1, 8], [5, 8, 8]]


def _ranges(cu, n_rows, max_new):
    """(first row, rows of a call, rows by the range) of every sequence, as the kernels bound them."""
    for a, b in zip(cu[:-1], cu[1:]):
        n = 0 if a < 0 else max(0, min(min(b, n_rows) - a, max_new))
        yield a, n, min(max(b - a, 0), 2 ** 31 - 1)


@pytest.mark.parametrize("layout", [TINY, B128, B96], ids=ids)
@pytest.mark.parametrize("cu", BAD_CU, ids=ids)
def test_row_ranges_that_are_none_touch_no_other_row_slot_or_score(layout, cu):
    """Row ranges that leave the arrays, run backwards or are longer than max_new: only rows that the arrays hold and that a
    range names are computed, and nothing around the arrays is written."""
    from paper_2601_19404_amd import binding as rpo
    Hq, Hkv, dh, dtype, pt = layout
    S, T, n, most = 2, 100, 8, 4
    c = Cache([T, T], Hkv, dh, pt, dtype, seed=1, stale=5.0)
    q, _, _ = _queries([n], Hq, dh, dtype, seed=1)
    dev = torch.tensor(cu, dtype=torch.int32).cuda()
    named = torch.zeros(n + 4, dtype=torch.bool)
    for a, k, _ in _ranges(cu, n, most):
        if k:
            named[2 + a: 2 + a + k] = True
    for use_ws in (False, True):
        guard = torch.full((n + 4, Hq * dh), 7.0, dtype=q.dtype, device="cuda")
        lse = torch.full((n + 4, Hq), 7.0, device="cuda")
        need = rpo.rpo_attn_paged_ws_bytes(c.dev, n, most, T, Hq) if use_ws else 0
        ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda") if need else None
        rpo.rpo_attn_paged(c.dev, q, dev, most, guard[2: 2 + n], lse_out_dev=lse[2: 2 + n], ws_dev=ws, max_len=T)
        torch.cuda.synchronize()
        assert torch.all(guard.cpu()[~named] == 7) and torch.all(lse.cpu()[~named] == 7)
        assert not (guard.cpu()[named] == 7).all(dim=1).any() and (ws is None or torch.all(ws[need:] == 255))
    score = torch.full((S + 2, Hkv, T + 5), 7.0, device="cuda")
    rpo.rpo_kv_score(c.dev, q, dev, most, lse[2: 2 + n].clone(), None, score[1: 1 + S], max_len=T)
    torch.cuda.synchronize()
    assert torch.all(score[0] == 7) and torch.all(score[1 + S] == 7) and torch.all(score[:, :, T:] == 7)
    want = c.pool.cpu().clone()
    for s, (a, k, by_range) in enumerate(_ranges(cu, n, most)):
        slots = torch.arange(T - by_range, T - by_range + k)
        keep = slots >= 0
        rows = q.cpu()[a: a + k][keep, : Hkv * dh].view(-1, Hkv, dh) if k else torch.zeros(0, Hkv, dh, dtype=q.dtype)
        c.write(want, s, slots[keep], rows, rows)
    rpo.rpo_kv_append(c.dev, q[:, : Hkv * dh], q[:, : Hkv * dh], dev, most)
    torch.cuda.synchronize()
    assert torch.equal(c.pool.cpu(), want)


@pytest.mark.parametrize("budget", [10, 100, 395])
def test_scores_of_kept_tokens_come_over_bit_for_bit(budget):
    """Zeros of both signs, infinities, numbers below the normal range and NaN."""
    from paper_2601_19404_amd import binding as rpo
    values = torch.tensor([0.0, -0.0, 1.0, -1.0, float("inf"), float("-inf"), float("nan"), 1e-42, -1e-42, 3e38])
    score = values[torch.randint(0, 10, (3, 2, 402), generator=torch.Generator().manual_seed(0))].cuda()
    c = Cache([400, 399, 120], 2, 32, 16, "f32", seed=1)
    to = Cache([0] * 3, 2, 32, 16, "f32", seed=2, cap=budget)
    kept, got = torch.zeros(3, 2, budget, dtype=torch.int32, device="cuda"), torch.full((3, 2, budget + 2), 7.0, device="cuda")
    rpo.rpo_kv_evict(c.dev, score, budget, 3, 4, to.dev, to.dev.lens, kept, got)
    torch.cuda.synchronize()
    for s in range(3):
        for h in range(2):
            slots = [j for j in kept[s, h].tolist() if j >= 0]
            assert torch.equal(got[s, h, : len(slots)].view(torch.int32), score[s, h, slots].view(torch.int32))
            assert torch.all(got[s, h, len(slots):] == 0)


@pytest.mark.parametrize("T", [4095, 4096, 4097, 16384, 16385, 32768, 32769])
def test_eviction_at_the_lengths_where_its_kernels_change(T):
    from paper_2601_19404_amd import binding as rpo
    budget, sinks, recent = 500, 4, 50
    c = Cache([T], 1, 32, 64, "bf16", seed=1, cap=T)
    to = Cache([0], 1, 32, 64, "bf16", seed=2, cap=budget, stale=0.0)
    score = torch.round(4 * torch.rand(1, 1, T, generator=torch.Generator().manual_seed(T))) / 4
    kept = torch.zeros(1, 1, budget, dtype=torch.int32, device="cuda")
    rpo.rpo_kv_evict(c.dev, score.cuda(), budget, sinks, recent, to.dev, to.dev.lens, kept)
    assert kept[0, 0].tolist() == O.evict(score[0, 0].numpy().astype(np.float64), budget, sinks, recent)


def test_eviction_into_free_pages_of_the_same_pool():
    """Source and target share the pool and the array of lengths, as a program with one pool has it."""
    from paper_2601_19404_amd import binding as rpo
    _, Hkv, dh, dtype, pt = B128
    lens, budget = [300, 65, 128], 70
    c = Cache(lens, Hkv, dh, pt, dtype, seed=1)
    free = torch.cat([c.pool, torch.full((6, c.pool.shape[1]), 3.0, dtype=c.pool.dtype, device="cuda")])
    n0 = c.pool.shape[0]
    src = rpo.PagedKV(free, c.dev.table, c.dev.lens, pt, Hkv, dh)
    table = torch.arange(n0, n0 + 6, dtype=torch.int32).view(3, 2).flip(0).contiguous()
    dst = rpo.PagedKV(free, table.cuda(), c.dev.lens, pt, Hkv, dh)
    score = torch.rand(3, Hkv, 300, generator=torch.Generator().manual_seed(1))
    kept = torch.zeros(3, Hkv, budget, dtype=torch.int32, device="cuda")
    rpo.rpo_kv_evict(src, score.cuda(), budget, 4, 16, dst, c.dev.lens, kept)
    torch.cuda.synchronize()
    assert torch.equal(free[:n0].view(torch.uint8), c.pool.view(torch.uint8)) and c.dev.lens.tolist() == [70, 65, 70]
    want = torch.full((n0 + 6, c.pool.shape[1]), 3.0, dtype=c.pool.dtype)
    c.table = table
    for s, T in enumerate(lens):
        for h in range(Hkv):
            slots = O.evict(score[s, h, :T].numpy().astype(np.float64), budget, 4, 16)
            c.write(want, s, torch.arange(len(slots)), c.k[s][slots, h], c.v[s][slots, h], h)
    assert torch.equal(free[n0:].cpu(), want[n0:])


@pytest.mark.parametrize("layout", [B128, F128], ids=ids)
@pytest.mark.parametrize("new", [1, 150])
def test_split_calls_are_captured_and_replayed(layout, new):
    """Attention and scores with workspaces that they need, in one graph; the rows' inputs and the lengths change between the
    replays, eager calls and another stream run in between: the eager results every time."""
    from paper_2601_19404_amd import binding as rpo
    Hq, Hkv, dh, dtype, pt = layout
    most = 3000
    c = Cache([most, 2100], Hkv, dh, pt, dtype, seed=1)
    q, cu, _ = _queries([new, new], Hq, dh, dtype, seed=1)
    q = q.clone()
    sizes = [f(c.dev, 2 * new, new, most, Hq) for f in (rpo.rpo_attn_paged_ws_bytes, rpo.rpo_kv_score_ws_bytes)]
    assert sizes[0] > 0 and (new == 1 or sizes[1] > 0)
    out, lse, score = torch.zeros_like(q), torch.zeros(2 * new, Hq, device="cuda"), torch.zeros(2, Hkv, most, device="cuda")

    def work(ws):
        rpo.rpo_attn_paged(c.dev, q, cu, new, out, lse_out_dev=lse, ws_dev=ws[0], max_len=most)
        rpo.rpo_kv_score(c.dev, q, cu, new, lse, None, score, ws_dev=ws[1], max_len=most)

    def run(call):
        for t in (out, lse, score):
            t.zero_()
        call()
        torch.cuda.synchronize()
        return [t.clone() for t in (out, lse, score)]

    spaces = [[torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None for n in sizes] for _ in range(3)]
    run(lambda: work(spaces[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(spaces[1])
    for lens in ([3000, 2100], [700, 2100], [2999, 1], [3000, 2047]):
        q.copy_(2 * torch.randn_like(q.float()))
        c.dev.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        want = run(lambda: work(spaces[0]))
        assert all(torch.equal(a, b) for a, b in zip(run(graph.replay), want)), lens

        def aside():
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                work(spaces[2])
        assert all(torch.equal(a, b) for a, b in zip(run(aside), want)), lens


def test_a_captured_decode_step_goes_on_by_itself():
    """Append, attention and scores of one step in a graph that counts the lengths up itself, replayed token after token."""
    from paper_2601_19404_amd import binding as rpo
    Hq, Hkv, dh, dtype, pt = B128
    start, steps = [60, 1000], 8
    make = lambda: Cache([0, 0], Hkv, dh, pt, dtype, seed=1, cap=1100, stale=0.25)   # noqa: E731
    rows = torch.randn(steps, 2, (Hq + 2 * Hkv) * dh, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    cu = torch.arange(3, dtype=torch.int32, device="cuda")
    results = []
    for captured in (False, True):
        c = make()
        c.dev.lens.copy_(torch.tensor(start, dtype=torch.int32))
        row, out, lse = rows[0].clone(), torch.zeros(2, Hq * dh, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, Hq, device="cuda")
        score = torch.zeros(2, Hkv, 1100, device="cuda")
        need = rpo.rpo_attn_paged_ws_bytes(c.dev, 2, 1, 1100, Hq)
        assert need > 0
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")

        def step():
            c.dev.lens.add_(1)
            rpo.rpo_kv_append(c.dev, row[:, Hq * dh: (Hq + Hkv) * dh], row[:, (Hq + Hkv) * dh:], cu, 1)
            rpo.rpo_attn_paged(c.dev, row[:, : Hq * dh], cu, 1, out, lse_out_dev=lse, ws_dev=ws, max_len=1100)
            rpo.rpo_kv_score(c.dev, row[:, : Hq * dh], cu, 1, lse, score, score, max_len=1100)

        call = step
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            call = graph.replay
        seen = []
        for i in range(steps):
            row.copy_(rows[i])
            call()
            torch.cuda.synchronize()
            seen.append((out.clone(), lse.clone(), score.clone()))
        assert c.dev.lens.tolist() == [n + steps for n in start]
        results.append((seen, c.pool))
    assert torch.equal(results[0][1], results[1][1])
    for a, b in zip(results[0][0], results[1][0]):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("layout", [TINY, B128, B64, F128, B32, B96], ids=ids)
@pytest.mark.parametrize("lens,new", [([130, 70], 2), ([130, 70], 60), ([1500, 900], 150), ([1500, 33], 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (25, 3)])
def test_values_reach_the_rows_that_see_them_and_no_others(layout, lens, new, window, sinks):
    """NaN and infinities in the values of tokens that some rows of a chunk see and others do not (the newest ones, and those that
    leave the window): the others come out as the oracle has them without, the log-sum-exp and the other heads bit for bit."""
    Hq, Hkv, dh, dtype, pt = layout
    news = [new, min(new, 33)]
    c = Cache(lens, Hkv, dh, pt, dtype, seed=2)
    q, cu, at = _queries(news, Hq, dh, dtype, seed=3)
    clean = [_attend(c, q, cu, new, Hq, window, sinks, use_ws) for use_ws in (False, True)]
    h, hpk = Hkv - 1, Hq // Hkv                                    # of the last KV head
    refs, bad = [], []                                             # bad: (sequence, slot, channel, value)
    for s, (T, n) in enumerate(zip(lens, news)):
        rows = q[at[s]: at[s + 1]].float().cpu().numpy().reshape(n, Hq, dh)[:, h * hpk:]
        refs.append(O.attention(rows, c.k[s][:, h:].float().numpy(), c.v[s][:, h:].float().numpy(), dh ** -0.5, window, sinks))
        bad += [(s, T - 1, 1, np.nan), (s, T - n // 2 - 1, 0, -np.inf), (s, T - n // 2, 2, np.inf), (s, T - n // 2, 3, np.nan)]
        leaves = T - n - window + 1 + n // 2                       # slot that only the first rows see
        if window and leaves >= sinks:
            bad += [(s, leaves, dh - 1, np.inf), (s, leaves, dh - 2, -np.inf)]
    for s, j, d, x in bad:
        v = c.v[s][j:j + 1].clone()
        v[:, h, d] = float(x)
        _rewrite(c, s, [j], v=v)
    for (want, want_lse), use_ws in zip(clean, (False, True)):
        out, lse = _attend(c, q, cu, new, Hq, window, sinks, use_ws)
        assert torch.equal(lse, want_lse) and torch.equal(out[:, : h * hpk * dh], want[:, : h * hpk * dh])
        for s, (T, n) in enumerate(zip(lens, news)):
            ref, _, _, mag, big = refs[s]
            got = out[at[s]: at[s + 1]].float().cpu().numpy().reshape(n, Hq, dh)[:, h * hpk:]
            expect = np.zeros((n, dh))
            t = np.arange(T - n, T)
            for s2, j, d, x in bad:
                if s2 == s:
                    sees = (j <= t) & ((t - j < window) | (j < sinks) | (window == 0))
                    with np.errstate(invalid="ignore"):
                        expect[:, d] += np.where(sees, x, 0.0)
            expect = np.broadcast_to(expect[:, None], got.shape)
            odd = ~np.isfinite(expect)
            np.testing.assert_array_equal(got[odd], expect[odd])
            assert np.all(np.isfinite(got[~odd]))
            off = np.abs(np.where(odd, 0.0, got) - np.where(odd, 0.0, ref)) - _chunk_tolerance(T, dh, ref, mag, big, dtype)
            assert off[~odd].max() <= 0, (s, use_ws, off[~odd].max())


@pytest.mark.parametrize("dtype,tokens", [("bf16", 1 << 24), ("f32", 1 << 23)])
def test_pages_so_long_that_a_slots_offset_passes_32_bits(dtype, tokens):
    """A cache in one page (two blocks of 4 GiB): rows at its end, whose keys and values lie more than 2^31 bytes into a block."""
    from paper_2601_19404_amd import binding as rpo
    Hq, Hkv, dh, near = 4, 1, 128, 300
    small = Cache([near], Hkv, dh, 64, dtype, seed=3)
    pool = torch.empty(1, 2 * tokens * dh, dtype=small.pool.dtype, device="cuda")
    length = tokens - 77
    lens, table = torch.tensor([length], dtype=torch.int32).cuda(), torch.zeros(1, 1, dtype=torch.int32).cuda()
    kv = rpo.PagedKV(pool, table, lens, tokens, Hkv, dh)
    k, v = (x[0].reshape(near, -1).cuda() for x in (small.k, small.v))
    rpo.rpo_kv_append(kv, k, v, torch.tensor([0, near], dtype=torch.int32).cuda(), near)
    for new in (1, 40):
        q, cu, _ = _queries([new], Hq, dh, dtype, seed=5)
        rows = q.float().cpu().numpy().reshape(new, Hq, dh)
        ref, _, p, mag, big = O.attention(rows, small.k[0].float().numpy(), small.v[0].float().numpy(), dh ** -0.5, 100)
        need = rpo.rpo_attn_paged_ws_bytes(kv, new, new, length, Hq, 100)
        out, lse = torch.zeros_like(q), torch.zeros(new, Hq, device="cuda")
        rpo.rpo_attn_paged(kv, q, cu, new, out, 100, lse_out_dev=lse, ws_dev=torch.empty(need, dtype=torch.uint8, device="cuda") if need else None,
                           max_len=length)
        score = torch.zeros(1, Hkv, length, device="cuda")
        rpo.rpo_kv_score(kv, q, cu, new, lse, None, score, 100, max_len=length)
        torch.cuda.synchronize()
        off = np.abs(out.float().cpu().numpy().reshape(ref.shape) - ref) - _chunk_tolerance(near, dh, ref, mag, big, dtype)
        assert off.max() <= 0, (new, off.max())
        assert torch.all(score[:, :, : length - near] == 0)
        w = O.score(p, Hkv)
        rel = EPS * (2 * ((dh + 10) * big.max() + near + 16) + new * Hq + 16)      # as in the other tests of the scores
        assert np.all(np.abs(score[0, :, length - near:].cpu().numpy() - w) <= rel * w + 2 * EPS * np.abs(w))


@pytest.mark.parametrize("layout", [TINY, B128, B64, F128, B96], ids=ids)
@pytest.mark.parametrize("new", [1, 8, 150])
@pytest.mark.parametrize("use_ws", [False, True])
def test_outputs_do_not_depend_on_whether_the_lse_is_asked_for(layout, new, use_ws):
    from paper_2601_19404_amd import binding as rpo
    Hq, Hkv, dh, dtype, pt = layout
    c = Cache([1500, 400], Hkv, dh, pt, dtype, seed=2)
    q, cu, _ = _queries([new, new], Hq, dh, dtype, seed=3)
    for window, sinks in ((0, 0), (700, 4)):
        want, _ = _attend(c, q, cu, new, Hq, window, sinks, use_ws)
        need = rpo.rpo_attn_paged_ws_bytes(c.dev, 2 * new, new, 1500, Hq, window, sinks) if use_ws else 0
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        out = torch.full_like(want, 7.0)
        rpo.rpo_attn_paged(c.dev, q, cu, new, out, window, sinks, ws_dev=ws, max_len=1500)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
