"""The paged-cache operators (append, attention with a window and sinks, weight scores, eviction) against the fp64 oracle.

Tolerances count roundings.  With eps = 2^-24 (fp32) every score has an error of at most (dh + 4) eps S, S the largest
scale sum |q_d k_jd| of a row, its exponential one of that and some 8 eps more, a sum of T terms T eps: together
r = eps ((dh + 10) S + T + 16) relative, on the weights and on their sum.  The bf16 path rounds the weights once
(2^-8 of sum p |v|) and the result once (2^-8 of the result)."""
import numpy as np
import pytest
import torch

from oracle import paged_kv as O

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


class Cache:
    """A cache filled from dense keys and values, its pages in random order among others that hold NaN."""

    def __init__(self, lens, Hkv, dh, pt, dtype, seed, cap=None, stale=float("nan"), stride_extra=0):
        from paper_2601_19404_amd import binding as rpo
        rng = np.random.default_rng(seed)
        dt = DT[dtype]
        per = max(1, -(-max(list(lens) + [cap or 0]) // pt))
        n_pages = len(lens) * per + 2
        self.Hkv, self.dh, self.pt, self.lens = Hkv, dh, pt, list(lens)
        self.k = [torch.from_numpy(rng.standard_normal((n, Hkv, dh)).astype(np.float32)).to(dt) for n in lens]
        self.v = [torch.from_numpy(rng.standard_normal((n, Hkv, dh)).astype(np.float32)).to(dt) for n in lens]
        size = 2 * Hkv * pt * dh
        pool = torch.full((n_pages, size + stride_extra), stale, dtype=dt)
        self.table = torch.from_numpy(rng.permutation(n_pages)[: len(lens) * per].astype(np.int32)).view(len(lens), per)
        for s, n in enumerate(lens):
            self.write(pool, s, torch.arange(n), self.k[s], self.v[s])
        self.pool = pool.cuda()
        self.dev = rpo.PagedKV(self.pool, self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(), pt, Hkv, dh)

    def views(self, pool):
        size = self.Hkv * self.pt * self.dh
        return (pool[:, :size].view(-1, self.Hkv, self.pt, self.dh),
                pool[:, size:2 * size].view(-1, self.Hkv, self.pt // 8, self.dh, 8))

    def write(self, pool, s, slots, k, v, h=slice(None)):
        """Keys and values of slots of a sequence, of all KV heads or of head h, into a pool of this cache's layout."""
        K, V = self.views(pool)
        page, at = self.table[s, slots // self.pt].long(), slots % self.pt
        K[page, h, at] = k
        V[page, h, at // 8, :, at % 8] = v

    def read(self, s, slots, h):
        """(keys, values) of a KV head's slots as they lie in the device's pool."""
        K, V = self.views(self.pool.cpu())
        page = self.table[s].long()[torch.as_tensor(slots) // self.pt]
        at = torch.as_tensor(slots) % self.pt
        return K[page, h, at], V[page, h, at // 8, :, at % 8]


def _queries(news, Hq, dh, dtype, seed, spread=2.0, extra=0, behind=0):
    """q with `extra` columns behind each row and `behind` rows behind the last sequence's."""
    g = torch.Generator().manual_seed(seed)
    n = sum(news) + behind
    wide = (spread * torch.randn(n, Hq * dh + extra, generator=g)).to(DT[dtype])
    cu = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32)
    return wide.cuda()[:, : Hq * dh], cu.cuda(), cu.tolist()


def _tolerance(T, dh, ref, mag, big, dtype):
    r = EPS * ((dh + 10) * big + T + 16)
    tol = 2 * r[..., None] * mag + EPS * np.abs(ref) + 1e-30
    return tol if dtype == "f32" else tol + 2.0 ** -8 * (mag + np.abs(ref)) * (1 + 2.0 ** -7)


def _check_attention(c, q, cu, news, Hq, window, sinks, dtype, use_ws, there=None, lens=None, max_len=None, stream=None):
    from paper_2601_19404_amd import binding as rpo
    lens = c.lens if lens is None else lens
    n, longest = q.shape[0], max(max(lens), 1) if max_len is None else max_len
    most = max(news)
    need = rpo.rpo_attn_paged_ws_bytes(c.dev, n, most, longest, Hq, window, sinks) if use_ws else 0
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    wide = torch.full((n, Hq * c.dh + 8), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((n, Hq), 7.0, device="cuda")
    rpo.rpo_attn_paged(c.dev, q, cu, most, wide[:, : Hq * c.dh], window, sinks, None, lse, ws, longest, stream)
    torch.cuda.synchronize()
    got, got_lse = wide.float().cpu().numpy(), lse.cpu().numpy()
    first = np.concatenate([[0], np.cumsum(news)])
    assert np.all(got[:, Hq * c.dh:] == 7) and np.all(got[first[-1]:] == 7) and np.all(got_lse[first[-1]:] == 7)
    weights = []
    for s in range(len(lens)):
        a, b = first[s], first[s + 1]
        qs = q[a:b].float().cpu().numpy().reshape(b - a, Hq, c.dh)
        T = lens[s]
        ref, ref_lse, p, mag, big = O.attention(qs, c.k[s][:T].float().numpy(), c.v[s][:T].float().numpy(), c.dh ** -0.5,
                                                window, sinks, None if there is None else there[s])
        weights.append(p)
        if a == b:
            continue
        x = got[a:b, : Hq * c.dh].reshape(ref.shape)
        off = np.abs(x - ref) - _tolerance(T, c.dh, ref, mag, big, dtype)
        assert np.all(np.isfinite(x)) and off.max() <= 0, f"sequence {s}: out {off.max():.3g} above its bound"
        some = np.isfinite(ref_lse)
        np.testing.assert_array_equal(np.isneginf(got_lse[a:b]), ~some)
        bound = EPS * ((c.dh + 10) * big + T + 16) + 2 * EPS * np.abs(np.where(some, ref_lse, 0.0)) + 8 * EPS
        d = np.abs(np.where(some, got_lse[a:b], 0.0) - np.where(some, ref_lse, 0.0)) - bound
        assert d.max() <= 0, f"sequence {s}: lse {d.max():.3g} above its bound"
        assert np.all(x[~some] == 0)
    return lse, weights


def _check_score(c, q, cu, news, Hq, window, sinks, lse, weights, use_ws=False, in_place=False, stride_extra=3, lens=None):
    from paper_2601_19404_amd import binding as rpo
    lens = c.lens if lens is None else lens
    longest = max(max(lens), 1)
    g = torch.Generator().manual_seed(5)
    before = torch.rand(len(lens), c.Hkv, longest + stride_extra, generator=g)
    src = before.cuda()
    dst = src if in_place else torch.full_like(src, -3.0)
    need = rpo.rpo_kv_score_ws_bytes(c.dev, q.shape[0], max(news), longest, Hq, window, sinks) if use_ws else 0
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    rpo.rpo_kv_score(c.dev, q, cu, max(news), lse, src, dst, window, sinks, None, ws, longest)
    torch.cuda.synchronize()
    got = dst.cpu().numpy()
    for s, T in enumerate(lens):
        rest = before[s, :, T:].numpy() if in_place else -3.0
        assert np.all(got[s, :, T:] == rest)
        p = weights[s]
        if p.shape[0] and T:
            rows = q[int(cu[s]): int(cu[s + 1])].float().cpu().numpy().reshape(p.shape[0], Hq, c.dh)
            big = np.abs(rows).max() * c.k[s][:T].float().abs().max().item() * c.dh * c.dh ** -0.5
            # twice r (the score and the lse it is compared with), one sum over rows and heads, the old value added
            rel = EPS * (2 * ((c.dh + 10) * big + T + 16) + p.shape[0] * Hq + 16)
            w = O.score(p, c.Hkv)
        else:
            rel, w = 0.0, np.zeros((c.Hkv, T))
        ref = before[s, :, :T].numpy().astype(np.float64) + w
        off = np.abs(got[s, :, :T] - ref) - (rel * w + 2 * EPS * np.abs(ref))
        assert T == 0 or off.max() <= 0, f"sequence {s}: score {off.max():.3g} above its bound"
    return dst


# head layouts: query heads, KV heads, channels, element type, page tokens
LAYOUTS = [(4, 2, 32, "f32", 16), (12, 2, 128, "bf16", 64), (28, 4, 128, "bf16", 64), (16, 4, 64, "bf16", 32),
           (6, 1, 128, "f32", 64), (2, 2, 128, "bf16", 16), (3, 3, 64, "f32", 128), (64, 1, 64, "bf16", 256),
           (4, 1, 32, "bf16", 16), (5, 1, 96, "bf16", 16), (2, 1, 256, "f32", 32), (2, 2, 2, "bf16", 16), (200, 1, 64, "bf16", 64)]
# lengths, new rows, window, sinks
SHAPES = [([1], [1], 0, 0), ([65, 1, 200], [1, 1, 1], 0, 0), ([130, 0, 17, 64, 63], [1, 0, 1, 1, 1], 20, 4),
          ([100, 33, 257], [100, 33, 257], 0, 0), ([150, 70, 5], [37, 70, 5], 16, 3), ([300, 300], [5, 2], 0, 0),
          ([190, 300, 64], [190, 3, 64], 1, 0), ([260, 90], [260, 1], 70, 100), ([310], [150], 1000, 4)]


@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda x: "-".join(map(str, x)))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda x: "-".join(map(str, x)).replace(" ", ""))
def test_attention_and_score(layout, shape):
    Hq, Hkv, dh, dtype, pt = layout
    lens, news, window, sinks = shape
    print(layout, shape, flush=True)
    c = Cache(lens, Hkv, dh, pt, dtype, seed=len(lens) + dh, stride_extra=8)
    q, cu, _ = _queries(news, Hq, dh, dtype, seed=dh, extra=8, behind=2)
    for use_ws in (False, True):
        lse, weights = _check_attention(c, q, cu, news, Hq, window, sinks, dtype, use_ws)
        _check_score(c, q, cu, news, Hq, window, sinks, lse, weights, use_ws, in_place=use_ws)


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[1], LAYOUTS[3], LAYOUTS[4]], ids=lambda x: "-".join(map(str, x)))
@pytest.mark.parametrize("new", [1, 2, 70])
@pytest.mark.parametrize("window,sinks", [(0, 0), (500, 4)])
def test_long_caches_split(layout, new, window, sinks):
    """Few rows over long caches: the tokens are split and the pieces joined; without a workspace they are not."""
    Hq, Hkv, dh, dtype, pt = layout
    lens, news = [2500, 1403], [new, min(new, 3)]
    c = Cache(lens, Hkv, dh, pt, dtype, seed=9)
    q, cu, _ = _queries(news, Hq, dh, dtype, seed=10)
    for use_ws in (True, False):
        lse, weights = _check_attention(c, q, cu, news, Hq, window, sinks, dtype, use_ws)
        _check_score(c, q, cu, news, Hq, window, sinks, lse, weights, use_ws)


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[1], LAYOUTS[9]], ids=lambda x: "-".join(map(str, x)))
def test_rows_below_slot_zero_and_pages_outside_the_pool(layout):
    """More rows than the cache has tokens: the first ones see nothing.  Table entries outside the pool: their tokens are
    not there, for attention and scores alike."""
    Hq, Hkv, dh, dtype, pt = layout
    lens, news = [3, 4 * pt + 5, 2 * pt], [9, 40, 1]
    c = Cache(lens, Hkv, dh, pt, dtype, seed=4)
    there = [np.ones(n, dtype=bool) for n in lens]
    c.table[1, 1], c.table[1, 3], c.table[2, 0], c.table[2, 1] = -1, c.pool.shape[0], 1 << 30, -(1 << 31)
    there[1][pt:2 * pt] = there[1][3 * pt:4 * pt] = there[2][:] = False
    c.dev.table.copy_(c.table)
    q, cu, _ = _queries(news, Hq, dh, dtype, seed=3)
    for window, sinks in ((0, 0), (pt + 3, 2)):
        lse, weights = _check_attention(c, q, cu, news, Hq, window, sinks, dtype, True, there)
        _check_score(c, q, cu, news, Hq, window, sinks, lse, weights)


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[1], LAYOUTS[9]], ids=lambda x: "-".join(map(str, x)))
def test_what_no_row_sees_may_be_nan(layout):
    """Tokens that a window hides from every row of the call, and everything beyond the length, hold NaN and infinities."""
    Hq, Hkv, dh, dtype, pt = layout
    lens, news, window, sinks = [200, 150], [1, 5], 30, 2
    c = Cache(lens, Hkv, dh, pt, dtype, seed=6)
    for s, n in enumerate(lens):
        pool, slots = c.pool.cpu(), torch.arange(sinks, n - news[s] + 1 - window)
        bad = torch.full((len(slots), Hkv, dh), float("nan"))
        bad[::2] = float("inf")
        c.write(pool, s, slots, bad.to(pool.dtype), -bad.flip(0).to(pool.dtype))
        c.pool.copy_(pool)
    q, cu, _ = _queries(news, Hq, dh, dtype, seed=3)
    for use_ws in (False, True):
        lse, weights = _check_attention(c, q, cu, news, Hq, window, sinks, dtype, use_ws)
        _check_score(c, q, cu, news, Hq, window, sinks, lse, weights)


def test_lengths_and_row_counts_beyond_what_the_arrays_hold_are_bounded():
    """A length past the table counts up to its end; rows past the row arrays and past max_new are not looked at."""
    from paper_2601_19404_amd import binding as rpo
    c = Cache([128, 128], 2, 128, 64, "bf16", seed=1)
    c.dev.lens.copy_(torch.tensor([1000, -5], dtype=torch.int32))
    q, _, _ = _queries([4, 4], 12, 128, "bf16", seed=1)
    cu = torch.tensor([0, 4, 8], dtype=torch.int32).cuda()
    _check_attention(c, q, cu, [4, 4], 12, 0, 0, "bf16", True, lens=[128, 0], max_len=128)
    out = torch.full_like(q, 7.0)
    for cu in ([0, 40, 80], [-3, 1, 2], [6, 2, 1 << 30], [9, 9, 9]):
        rpo.rpo_attn_paged(c.dev, q, torch.tensor(cu, dtype=torch.int32).cuda(), 4, out)
    torch.cuda.synchronize()
    assert out.shape[0] == 8


def test_equal_inputs_give_equal_bits_and_shared_pages_equal_rows():
    from paper_2601_19404_amd import binding as rpo
    c = Cache([700, 700], 2, 128, 64, "bf16", seed=2)
    c.dev.table[1] = c.dev.table[0]
    q, cu, _ = _queries([3, 3], 12, 128, "bf16", seed=2)
    q = q.clone()
    q[3:] = q[:3]
    need = rpo.rpo_attn_paged_ws_bytes(c.dev, 6, 3, 700, 12)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    got = []
    for _ in range(3):
        out, lse = torch.zeros_like(q), torch.zeros(6, 12, device="cuda")
        score = torch.zeros(2, 2, 700, device="cuda")
        rpo.rpo_attn_paged(c.dev, q, cu, 3, out, lse_out_dev=lse, ws_dev=ws, max_len=700)
        rpo.rpo_kv_score(c.dev, q, cu, 3, lse, None, score, max_len=700)
        got.append((out, lse, score))
    for out, lse, score in got:
        assert torch.equal(out, got[0][0]) and torch.equal(lse, got[0][1]) and torch.equal(score, got[0][2])
        assert torch.equal(out[:3], out[3:]) and torch.equal(score[0], score[1])


# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[1], LAYOUTS[3], LAYOUTS[9], LAYOUTS[11]], ids=lambda x: "-".join(map(str, x)))
@pytest.mark.parametrize("lens,news", [([1, 40, 7], [1, 1, 1]), ([100, 33, 0, 257], [90, 33, 0, 13]), ([3, 64], [8, 64])])
def test_append(layout, lens, news):
    """The rows land in their slots, bit for bit, and nothing else of the pool changes; rows below slot 0 are dropped."""
    from paper_2601_19404_amd import binding as rpo
    _, Hkv, dh, dtype, pt = layout
    c = Cache(lens, Hkv, dh, pt, dtype, seed=3, stale=5.0)
    g = torch.Generator().manual_seed(1)
    wide = torch.randn(sum(news) + 1, 2 * Hkv * dh + 8, generator=g).to(DT[dtype])
    want = c.pool.cpu().clone()
    row = 0
    for s, (T, n) in enumerate(zip(lens, news)):
        low = max(0, n - T)                      # rows below slot 0
        rows = wide[row + low: row + n, : 2 * Hkv * dh].view(-1, 2, Hkv, dh)
        c.write(want, s, torch.arange(T - n + low, T), rows[:, 0], rows[:, 1])
        row += n
    cu = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32).cuda()
    for src in (wide.cuda(), torch.cat([wide[:, :1], wide], dim=1).cuda()[:, 1:]):   # aligned rows, and shifted by one element
        start = c.pool.clone()
        rpo.rpo_kv_append(c.dev, src[:, : Hkv * dh], src[:, Hkv * dh: 2 * Hkv * dh], cu, max(news))
        torch.cuda.synchronize()
        assert torch.equal(c.pool.cpu(), want)
        c.pool.copy_(start)


def _evict_case(lens, Hkv, dh, pt, dtype, budget, sinks, recent, seed, ties, dst_pt=None, score=None):
    from paper_2601_19404_amd import binding as rpo
    dst_pt = dst_pt or pt
    c = Cache(lens, Hkv, dh, pt, dtype, seed=seed)
    to = Cache([0] * len(lens), Hkv, dh, dst_pt, dtype, seed=seed + 1, cap=budget, stale=9.0)
    longest = max(max(lens), 1)
    if score is None:
        g = torch.Generator().manual_seed(seed)
        score = torch.exp(1.5 * torch.randn(len(lens), Hkv, longest + 2, generator=g))
        if ties:
            score = torch.round(score)
    kept = torch.full((len(lens), Hkv, budget), -7, dtype=torch.int32, device="cuda")
    new_score = torch.full((len(lens), Hkv, budget + 3), -7.0, device="cuda")
    src_before = c.pool.clone()
    rpo.rpo_kv_evict(c.dev, score.cuda(), budget, sinks, recent, to.dev, to.dev.lens, kept, new_score)
    torch.cuda.synchronize()
    assert torch.equal(c.pool.view(torch.uint8), src_before.view(torch.uint8))
    assert to.dev.lens.tolist() == [min(n, budget) for n in lens]
    want = torch.full_like(to.pool, 9.0).cpu()
    for s, T in enumerate(lens):
        for h in range(Hkv):
            slots = O.evict(score[s, h, :T].numpy().astype(np.float64), budget, sinks, recent)
            got = kept[s, h].tolist()
            assert got == slots + [-1] * (budget - len(slots)), f"sequence {s}, head {h}"
            assert torch.equal(new_score[s, h, : len(slots)].cpu(), score[s, h, slots]) or score.isnan().any()
            assert torch.all(new_score[s, h, len(slots):] == 0)
            to.write(want, s, torch.arange(len(slots)), c.k[s][slots, h], c.v[s][slots, h], h)
    assert torch.equal(to.pool.cpu(), want)


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[1], LAYOUTS[3], LAYOUTS[9], LAYOUTS[11]], ids=lambda x: "-".join(map(str, x)))
@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (1, 1, 0), (50, 4, 20), (77, 0, 77), (64, 10, 0), (200, 3, 5), (300, 0, 0)])
@pytest.mark.parametrize("ties", [False, True])
def test_evict(layout, budget, sinks, recent, ties):
    _, Hkv, dh, dtype, pt = layout
    _evict_case([250, 0, 1, 77, 201, 64], Hkv, dh, pt, dtype, budget, sinks, recent, seed=budget, ties=ties,
                dst_pt=64 if pt == 16 else 16)


@pytest.mark.parametrize("T,budget,sinks,recent", [(5000, 1024, 4, 256), (5000, 4999, 0, 1), (20000, 37, 4, 0), (2049, 2048, 1, 1)])
@pytest.mark.parametrize("ties", [False, True])
def test_evict_long(T, budget, sinks, recent, ties):
    _evict_case([T, T - 1000], 2, 32, 64, "bf16", budget, sinks, recent, seed=T, ties=ties)


def test_evict_odd_scores():
    """Infinities, zeros of both signs, negative numbers, numbers below the normal range, and NaN, which ranks lowest."""
    values = torch.tensor([0.0, -0.0, 1.0, -1.0, float("inf"), float("-inf"), float("nan"), 1e-42, -1e-42, 3e38])
    g = torch.Generator().manual_seed(0)
    score = values[torch.randint(0, 10, (3, 2, 402), generator=g)]
    for budget in (10, 100, 395):
        _evict_case([400, 399, 120], 2, 32, 16, "f32", budget, 3, 4, seed=2, ties=False, score=score)
    _evict_case([400], 1, 32, 16, "f32", 64, 0, 0, seed=2, ties=False, score=torch.full((1, 1, 400), float("nan")))


def test_evict_lengths_in_place_of_the_sources():
    from paper_2601_19404_amd import binding as rpo
    c = Cache([100, 20], 2, 128, 64, "bf16", seed=1)
    to = Cache([0, 0], 2, 128, 64, "bf16", seed=2, cap=64, stale=0.0)
    score = torch.rand(2, 2, 100).cuda()
    kept = torch.zeros(2, 2, 33, dtype=torch.int32, device="cuda")
    rpo.rpo_kv_evict(c.dev, score, 33, 1, 1, to.dev, c.dev.lens, kept)
    assert c.dev.lens.tolist() == [33, 20]


# ---------------------------------------------------------------------------------------------
def test_rollout_with_a_bounded_cache():
    """The operators together, as a decode loop with a budget uses them: append, attend, score, evict when the cache is
    full, go on in the smaller cache.  The oracle does the same in fp64 with the slots that the GPU kept (each checked to
    be what the scores that the GPU had ask for)."""
    from paper_2601_19404_amd import binding as rpo
    Hq, Hkv, dh, pt, cap, budget, sinks, recent, S = 12, 2, 128, 64, 192, 96, 4, 32, 3
    rng = np.random.default_rng(0)
    draw = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).bfloat16()   # noqa: E731
    lens = [0] * S
    caches = [Cache([0] * S, Hkv, dh, pt, "bf16", seed=i, cap=cap) for i in range(2)]
    here = 0
    score = torch.zeros(S, Hkv, cap, device="cuda")
    dense = [[np.zeros((0, dh)), np.zeros((0, dh)), np.zeros(0)] for _ in range(S * Hkv)]      # keys, values, weights
    evictions = 0
    for step, news in enumerate([[150, 61, 100], [1, 1, 1], [40, 7, 0], [1, 1, 1], [30, 90, 80], [1, 1, 1], [1, 1, 1]]):
        c = caches[here]
        n = sum(news)
        q, k, v = 2 * draw(n, Hq * dh), draw(n, Hkv * dh), draw(n, Hkv * dh)
        cu = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32).cuda()
        lens = [a + b for a, b in zip(lens, news)]
        c.dev.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        out, lse = torch.zeros(n, Hq * dh, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, Hq, device="cuda")
        window = 80 if step % 2 else 0
        rpo.rpo_kv_append(c.dev, k.cuda(), v.cuda(), cu, max(news))
        rpo.rpo_attn_paged(c.dev, q.cuda(), cu, max(news), out, window, sinks, lse_out_dev=lse, max_len=max(lens))
        rpo.rpo_kv_score(c.dev, q.cuda(), cu, max(news), lse, score, score, window, sinks, max_len=max(lens))
        got, w = out.float().cpu().numpy(), score.cpu().numpy()
        at = np.concatenate([[0], np.cumsum(news)])
        for s in range(S):
            a, b = at[s], at[s + 1]
            for h in range(Hkv):
                d = dense[s * Hkv + h]
                d[0] = np.concatenate([d[0], k[a:b].float().numpy().reshape(-1, Hkv, dh)[:, h]])
                d[1] = np.concatenate([d[1], v[a:b].float().numpy().reshape(-1, Hkv, dh)[:, h]])
                qs = q[a:b].float().numpy().reshape(-1, Hkv, Hq // Hkv, dh)[:, h]
                ref, _, p, mag, big = O.attention(qs, d[0][:, None], d[1][:, None], dh ** -0.5, window, sinks)
                d[2] = np.concatenate([d[2], np.zeros(b - a)]) + O.score(p, 1)[0]
                if a < b:
                    x = got[a:b].reshape(-1, Hkv, Hq // Hkv, dh)[:, h]
                    assert np.all(np.abs(x - ref) <= _tolerance(lens[s], dh, ref, mag, big, "bf16")), (step, s, h)
                np.testing.assert_allclose(w[s, h, : lens[s]], d[2], rtol=1e-3, atol=1e-5)
        if max(lens) > cap - 2:
            evictions += 1
            to = caches[1 - here]
            kept = torch.zeros(S, Hkv, budget, dtype=torch.int32, device="cuda")
            new_score = torch.zeros(S, Hkv, cap, device="cuda")
            rpo.rpo_kv_evict(c.dev, score, budget, sinks, recent, to.dev, to.dev.lens, kept, new_score)
            for s in range(S):
                for h in range(Hkv):
                    slots = [j for j in kept[s, h].tolist() if j >= 0]
                    assert slots == O.evict(w[s, h, : lens[s]].astype(np.float64), budget, sinks, recent)
                    d = dense[s * Hkv + h]
                    d[0], d[1], d[2] = d[0][slots], d[1][slots], d[2][slots]
            lens = to.dev.lens.tolist()
            score, here = new_score, 1 - here
    assert evictions == 1          # 191 tokens in the third step; 96, 69 and 96 are left and grow to at most 179


def test_cache_of_a_batch_matches_its_decode_attention():
    """rpo_batch_kv's pages under rpo_attn_paged: without a window the same attention as rpo_attn_decode's."""
    from paper_2601_19404_amd import binding as rpo
    from paper_2601_19404_amd import synth
    from tests.util import to_device
    mc = synth.ModelCfg("1.5B-heads", 2, 256, 12, 2, 128, 512, 1000, "bf16")
    model = rpo.rpo_model_create(mc, to_device(synth.make_weights(mc)))
    n_groups, G, plen = 2, 4, [150, 201]
    batch = rpo.rpo_batch_create(model, n_groups, G, 256, 32, 64, 512)
    with pytest.raises(rpo.RpoError) as e:
        rpo.PagedKV.of_batch(batch, 0, torch.zeros(8, dtype=torch.int32, device="cuda"))
    assert e.value.code == rpo.RPO_ESTATE
    g = torch.Generator().manual_seed(0)
    toks = torch.randint(0, 1000, (sum(plen),), generator=g, dtype=torch.int32).cuda()
    logits = torch.zeros(n_groups, 1000, device="cuda")
    rpo.rpo_prefill_prefix(batch, toks, [0, 150, 351], logits)
    rpo.rpo_kv_fork(batch)
    step = torch.zeros(8, 1000, device="cuda")
    for j in range(3):
        rpo.rpo_decode_step(batch, torch.full((8,), 5 + j, dtype=torch.int32, device="cuda"), 8, None, step)
    q = torch.randn(8, 12 * 128, generator=g).to(torch.bfloat16).cuda()
    want, out = torch.zeros_like(q), torch.zeros_like(q)
    lens = torch.tensor([plen[r // G] + 3 for r in range(8)], dtype=torch.int32, device="cuda")
    cu = torch.arange(9, dtype=torch.int32, device="cuda")
    for layer in range(2):
        kv = rpo.PagedKV.of_batch(batch, layer, lens)
        rpo.rpo_attn_decode(batch, layer, q, 8, 3, None, want)
        rpo.rpo_attn_paged(kv, q, cu, 1, out)
        torch.cuda.synchronize()
        # two kernels that each round p and the result to bf16: 2 x 2 x 2^-8 of values below max |v|
        assert (want.float() - out.float()).abs().max() <= 4 * 2.0 ** -8 * want.float().abs().max()
    with pytest.raises(rpo.RpoError):
        rpo.PagedKV.of_batch(batch, 2, lens)


def test_captured_graphs_replay_and_other_streams():
    """Attention, score and eviction captured into one graph, replayed with other inputs, and the same calls on a stream of
    the program's own: the eager results every time."""
    from paper_2601_19404_amd import binding as rpo
    c = Cache([900, 650], 2, 128, 64, "bf16", seed=1)
    to = Cache([0, 0], 2, 128, 64, "bf16", seed=2, cap=128, stale=0.0)
    q, cu, _ = _queries([1, 1], 12, 128, "bf16", seed=1)
    k = torch.randn(2, 256, device="cuda").bfloat16()
    need = rpo.rpo_attn_paged_ws_bytes(c.dev, 2, 1, 900, 12, 300, 4)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(2, 12, device="cuda")
    score, kept = torch.zeros(2, 2, 900, device="cuda"), torch.zeros(2, 2, 128, dtype=torch.int32, device="cuda")
    new_score, new_len = torch.zeros(2, 2, 128, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")

    def work():
        rpo.rpo_kv_append(c.dev, k, k, cu, 1)
        rpo.rpo_attn_paged(c.dev, q, cu, 1, out, 300, 4, lse_out_dev=lse, ws_dev=ws, max_len=900)
        rpo.rpo_kv_score(c.dev, q, cu, 1, lse, None, score, 300, 4, max_len=900)
        rpo.rpo_kv_evict(c.dev, score, 128, 4, 16, to.dev, new_len, kept, new_score)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (out, lse, score, kept, new_score, new_len, to.pool, c.pool.nan_to_num())]

    work()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        work()
    for i in range(3):
        q.copy_(2 * torch.randn_like(q.float()))
        k.copy_(torch.randn(2, 256, device="cuda"))
        for t in (out, lse, score, kept, new_score, new_len, to.pool):
            t.zero_()
        graph.replay()
        got = results()
        work()
        assert all(torch.equal(a, b) for a, b in zip(got, results())), f"replay {i}"
        side = torch.cuda.Stream()
        for t in (out, lse, score, kept, new_score, new_len, to.pool):
            t.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            work()
        assert all(torch.equal(a, b) for a, b in zip(got, results())), f"stream {i}"


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 bytes and elements' offsets beyond 2^31: pages at its end."""
    from paper_2601_19404_amd import binding as rpo
    Hq, Hkv, dh, pt = 12, 2, 128, 64
    size = 2 * Hkv * pt * dh
    n_pages = (1 << 32) // size + 100          # elements beyond 2^32
    pool = torch.empty(n_pages, size, dtype=torch.bfloat16, device="cuda")
    small = Cache([300], Hkv, dh, pt, "bf16", seed=5)
    table = torch.arange(n_pages - 5, n_pages, dtype=torch.int32).view(1, 5).cuda()
    kv = rpo.PagedKV(pool, table, small.dev.lens, pt, Hkv, dh)
    cu = torch.tensor([0, 300], dtype=torch.int32).cuda()
    k, v = (x[0].reshape(300, -1).cuda() for x in (small.k, small.v))
    rpo.rpo_kv_append(kv, k, v, cu, 300)
    q, cu, _ = _queries([20], Hq, dh, "bf16", seed=5)
    small.dev, small.pool = kv, pool
    lse, weights = _check_attention(small, q, cu, [20], Hq, 100, 4, "bf16", True)
    _check_score(small, q, cu, [20], Hq, 100, 4, lse, weights)
    to = Cache([0], Hkv, dh, pt, "bf16", seed=2, cap=128, stale=0.0)
    kept = torch.zeros(1, Hkv, 100, dtype=torch.int32, device="cuda")
    score = torch.rand(1, Hkv, 300, device="cuda")
    rpo.rpo_kv_evict(kv, score, 100, 4, 10, to.dev, to.dev.lens, kept)
    torch.cuda.synchronize()
    for h in range(Hkv):
        keys, values = to.read(0, list(range(100)), h)
        slots = kept[0, h].tolist()
        assert torch.equal(keys, small.k[0][slots, h]) and torch.equal(values, small.v[0][slots, h])


def test_binding_refuses_what_does_not_fit():
    from paper_2601_19404_amd import binding as rpo
    c = Cache([100], 2, 128, 64, "bf16", seed=1)
    q, cu, _ = _queries([2], 12, 128, "bf16", seed=1)
    out, lse = torch.zeros_like(q), torch.zeros(2, 12, device="cuda")
    score = torch.zeros(1, 2, 100, device="cuda")
    for call in (lambda: rpo.rpo_attn_paged(c.dev, q.float(), cu, 2, out),
                 lambda: rpo.rpo_attn_paged(c.dev, q, cu, 2, out[:1]),
                 lambda: rpo.rpo_attn_paged(c.dev, q.t().contiguous().t(), cu, 2, out),
                 lambda: rpo.rpo_attn_paged(c.dev, q, cu.long(), 2, out),
                 lambda: rpo.rpo_attn_paged(c.dev, q, cu[:1], 2, out),
                 lambda: rpo.rpo_attn_paged(c.dev, q, cu, 2, out, lse_out_dev=lse[:1]),
                 lambda: rpo.rpo_attn_paged(c.dev, q.cpu(), cu, 2, out),
                 lambda: rpo.rpo_attn_paged(c.dev, q[:, :1500], cu, 2, out[:, :1500]),
                 lambda: rpo.rpo_kv_score(c.dev, q, cu, 2, lse, score[:, :1], score),
                 lambda: rpo.rpo_kv_score(c.dev, q, cu, 2, lse, None, score[0]),
                 lambda: rpo.rpo_kv_append(c.dev, q[:, :256], q[:1, :256], cu, 2),
                 lambda: rpo.rpo_kv_append(c.dev, q, q, cu, 2),
                 lambda: rpo.rpo_kv_evict(c.dev, score, 50, 0, 0, c.dev, c.dev.lens, torch.zeros(10, dtype=torch.int32, device="cuda")),
                 lambda: rpo.PagedKV(c.pool, c.dev.table, c.dev.lens, 128, 2, 128),
                 lambda: rpo.PagedKV(c.pool, c.dev.table[0], c.dev.lens, 64, 2, 128)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: rpo.rpo_attn_paged(c.dev, q, cu, 3, out), lambda: rpo.rpo_attn_paged(c.dev, q, cu, 2, out, -1),
                 lambda: rpo.rpo_attn_paged(c.dev, q, cu, 2, out, scale=0.0)):
        with pytest.raises(rpo.RpoError) as e:
            call()
        assert e.value.code == rpo.RPO_EINVAL
    assert torch.all(out == 0)


@pytest.mark.parametrize("ties", [False, True])
def test_evict_rows_too_long_for_registers(ties):
    _evict_case([40000, 39000], 1, 32, 64, "bf16", 3000, 4, 100, seed=5, ties=ties)


def test_calls_without_rows_and_without_tokens():
    """No rows: attention does nothing, scores are copied; all caches empty: rows see nothing, nothing is kept."""
    from paper_2601_19404_amd import binding as rpo
    c = Cache([100, 30], 2, 128, 64, "bf16", seed=1)
    q = torch.zeros(0, 12 * 128, dtype=torch.bfloat16, device="cuda")
    cu = torch.zeros(3, dtype=torch.int32, device="cuda")
    before = torch.rand(2, 2, 100).cuda()
    after = torch.full_like(before, -1.0)
    rpo.rpo_attn_paged(c.dev, q, cu, 0, torch.zeros_like(q))
    rpo.rpo_kv_append(c.dev, q[:, :256], q[:, :256], cu, 0)
    rpo.rpo_kv_score(c.dev, q, cu, 0, torch.zeros(0, 12, device="cuda"), before, after)
    torch.cuda.synchronize()
    for s, n in enumerate((100, 30)):
        assert torch.equal(after[s, :, :n], before[s, :, :n]) and torch.all(after[s, :, n:] == -1)
    rows, cu2, _ = _queries([2, 20], 12, 128, "bf16", seed=1)
    c.dev.lens.zero_()
    _check_attention(c, rows, cu2, [2, 20], 12, 0, 0, "bf16", True, lens=[0, 0], max_len=0)
    to = Cache([0, 0], 2, 128, 64, "bf16", seed=2, cap=64, stale=3.0)
    kept = torch.full((2, 2, 50), 5, dtype=torch.int32, device="cuda")
    rpo.rpo_kv_evict(c.dev, before, 50, 0, 0, to.dev, to.dev.lens, kept)
    assert to.dev.lens.tolist() == [0, 0] and torch.all(kept == -1) and torch.all(to.pool == 3)


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[1], LAYOUTS[10]], ids=lambda x: "-".join(map(str, x)))
def test_the_largest_window_and_number_of_sinks(layout):
    """2^31 - 1 of either hides nothing, also from rows far below slot 0."""
    Hq, Hkv, dh, dtype, pt = layout
    lens, news, most = [70, 3], [70, 40], 2 ** 31 - 1
    c = Cache(lens, Hkv, dh, pt, dtype, seed=4)
    q, cu, _ = _queries(news, Hq, dh, dtype, seed=3)
    for window, sinks in ((most, 0), (most, most), (5, most)):
        lse, weights = _check_attention(c, q, cu, news, Hq, window, sinks, dtype, True)
        _check_score(c, q, cu, news, Hq, window, sinks, lse, weights)


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[1], LAYOUTS[4]], ids=lambda x: "-".join(map(str, x)))
@pytest.mark.parametrize("new", [1, 50])
def test_scores_that_climb_by_hundreds(layout, new):
    """Scores rise along the cache from far below to far above: the reference point of the weights has to move many times,
    and weights that are due already move with it."""
    Hq, Hkv, dh, dtype, pt = layout
    lens, news = [330, 100], [new, min(new, 100)]
    c = Cache(lens, Hkv, dh, pt, dtype, seed=8)
    pool = c.pool.cpu()
    for s, n in enumerate(lens):
        ramp = torch.linspace(-3.0, 3.0, n)[:, None, None] * torch.ones(1, Hkv, dh)
        c.k[s] = (ramp + 0.05 * c.k[s].float()).to(c.k[s].dtype)
        c.write(pool, s, torch.arange(n), c.k[s], c.v[s])
    c.pool.copy_(pool)
    q, cu, _ = _queries(news, Hq, dh, dtype, seed=3)
    q = (q.float().abs() + 2.0).to(q.dtype)          # scores of about -100 (32 channels) to 250 (128)
    for use_ws in (False, True):
        lse, weights = _check_attention(c, q, cu, news, Hq, 0, 0, dtype, use_ws)
        _check_score(c, q, cu, news, Hq, 0, 0, lse, weights)


def test_a_nan_in_a_query_stays_in_its_row():
    from paper_2601_19404_amd import binding as rpo
    c = Cache([200], 2, 128, 64, "bf16", seed=4)
    q, cu, _ = _queries([40], 12, 128, "bf16", seed=3)
    q = q.clone()
    want, lse = torch.zeros_like(q), torch.zeros(40, 12, device="cuda")
    rpo.rpo_attn_paged(c.dev, q, cu, 40, want, lse_out_dev=lse)
    q[7, 128:256] = float("nan")
    out, lse2 = torch.zeros_like(q), torch.zeros(40, 12, device="cuda")
    rpo.rpo_attn_paged(c.dev, q, cu, 40, out, lse_out_dev=lse2)
    torch.cuda.synchronize()
    assert out[7, 128:256].isnan().all() and lse2[7, 1].isnan()
    out[7, 128:256], lse2[7, 1] = want[7, 128:256], lse[7, 1]
    assert torch.equal(out, want) and torch.equal(lse, lse2)


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[1], LAYOUTS[3]], ids=lambda x: "-".join(map(str, x)))
def test_rows_off_16_bytes_and_the_generic_kernels(layout):
    """Query rows that start anywhere take the generic kernels, as everything does with kernel path 1."""
    from paper_2601_19404_amd import binding as rpo
    Hq, Hkv, dh, dtype, pt = layout
    lens, news, window, sinks = [150, 70], [37, 3], 40, 3
    c = Cache(lens, Hkv, dh, pt, dtype, seed=4)
    wide, cu, _ = _queries(news, Hq, dh, dtype, seed=3, extra=7)
    off = torch.cat([wide[:, :1], wide], dim=1)[:, 1:]
    assert off.data_ptr() % 16 and off.stride(0) * off.element_size() % 16
    for q, path in ((off, 0), (wide.contiguous(), 1)):
        rpo.rpo_set_kernel_path(path)
        try:
            lse, weights = _check_attention(c, q, cu, news, Hq, window, sinks, dtype, True)
            _check_score(c, q, cu, news, Hq, window, sinks, lse, weights, True)
        finally:
            rpo.rpo_set_kernel_path(0)


def test_two_calls_at_once_with_a_workspace_each():
    from paper_2601_19404_amd import binding as rpo
    streams, work, want = [torch.cuda.Stream() for _ in range(2)], [], []
    for i in range(2):
        c = Cache([3000, 1700], 2, 128, 64, "bf16", seed=i)
        q, cu, _ = _queries([2, 2], 12, 128, "bf16", seed=i)
        need = rpo.rpo_attn_paged_ws_bytes(c.dev, 4, 2, 3000, 12)
        assert need > 0
        work.append((c, q, cu, torch.zeros_like(q), torch.empty(need, dtype=torch.uint8, device="cuda")))
    for c, q, cu, out, ws in work:
        rpo.rpo_attn_paged(c.dev, q, cu, 2, out, ws_dev=ws, max_len=3000)
    torch.cuda.synchronize()
    want = [w[3].clone() for w in work]
    for w in work:
        w[3].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for (c, q, cu, out, ws), s in zip(work, streams):
            rpo.rpo_attn_paged(c.dev, q, cu, 2, out, ws_dev=ws, max_len=3000, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(w[3], x) for w, x in zip(work, want))


def test_a_batchs_cache_is_scored_and_evicted_into_pages_of_ones_own():
    """Prefill and fork a batch, score its prefix with queries of one's own, keep half of every rollout's cache and attend to
    what is left: the oracle's attention over the kept tokens of the batch's pages."""
    from paper_2601_19404_amd import binding as rpo
    from paper_2601_19404_amd import synth
    from tests.util import to_device
    mc = synth.ModelCfg("1.5B-heads", 1, 256, 12, 2, 128, 512, 1000, "bf16")
    model = rpo.rpo_model_create(mc, to_device(synth.make_weights(mc)))
    n_groups, G, plen = 2, 2, [150, 201]
    batch = rpo.rpo_batch_create(model, n_groups, G, 256, 32, 64, 512)
    g = torch.Generator().manual_seed(0)
    toks = torch.randint(0, 1000, (sum(plen),), generator=g, dtype=torch.int32).cuda()
    rpo.rpo_prefill_prefix(batch, toks, [0, 150, 351], torch.zeros(n_groups, 1000, device="cuda"))
    rpo.rpo_kv_fork(batch)
    lens = [plen[r // G] for r in range(4)]
    kv = rpo.PagedKV.of_batch(batch, 0, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    q, cu, _ = _queries([3] * 4, 12, 128, "bf16", seed=3)
    out, lse = torch.zeros_like(q), torch.zeros(12, 12, device="cuda")
    score = torch.zeros(4, 2, 201, device="cuda")
    pool_before = batch.kv_pool.clone()
    rpo.rpo_attn_paged(kv, q, cu, 3, out, lse_out_dev=lse)
    rpo.rpo_kv_score(kv, q, cu, 3, lse, None, score)
    budget = 90
    to = Cache([0] * 4, 2, 128, 64, "bf16", seed=2, cap=budget, stale=float("nan"))
    kept = torch.zeros(4, 2, budget, dtype=torch.int32, device="cuda")
    rpo.rpo_kv_evict(kv, score, budget, 4, 16, to.dev, to.dev.lens, kept)
    rpo.rpo_attn_paged(to.dev, q, cu, 3, out, lse_out_dev=lse)
    torch.cuda.synchronize()
    assert torch.equal(batch.kv_pool, pool_before) and to.dev.lens.tolist() == [budget] * 4
    w = score.cpu().numpy()
    assert np.allclose(w.sum(axis=(1, 2)), 3 * 12, rtol=1e-4)          # every row gives each of its heads' weights once
    pool = batch.kv_pool.view(torch.bfloat16).view(-1, 2, 2, 64 * 128).cpu()     # one layer
    pages = lambda r: [(r // G) * 4 + k if k < plen[r // G] // 64 else 2 * 4 + r * batch_private for k in range(-(-lens[r] // 64))]  # noqa: E731
    batch_private = -(-(64 - 1 + 32) // 64)
    got = out.float().cpu().numpy().reshape(4, 3, 12, 128)
    for r in range(4):
        K = torch.cat([pool[p, 0].view(2, 64, 128) for p in pages(r)], dim=1)
        V = torch.cat([pool[p, 1].view(2, 8, 128, 8).permute(0, 1, 3, 2).reshape(2, 64, 128) for p in pages(r)], dim=1)
        for h in range(2):
            slots = kept[r, h].tolist()
            assert slots == O.evict(w[r, h, : lens[r]].astype(np.float64), budget, 4, 16)
            keys, values = to.read(r, list(range(budget)), h)
            assert torch.equal(keys, K[h, slots]) and torch.equal(values, V[h, slots])
            rows = q[3 * r: 3 * r + 3].float().cpu().numpy().reshape(3, 2, 6, 128)[:, h]
            ref, _, p, mag, big = O.attention(rows, K[h, slots].float().numpy()[:, None], V[h, slots].float().numpy()[:, None], 128 ** -0.5)
            assert np.all(np.abs(got[r][:, 6 * h: 6 * h + 6] - ref) <= _tolerance(budget, 128, ref, mag, big, "bf16"))
