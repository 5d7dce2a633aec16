"""The operators of a bounded key/value cache, as cases that can be timed: new tokens written into pages (append),
attention of a chunk of new tokens or of single tokens over the pages, with a sliding window and sinks (attn), the
attention weight that every cached token has received (score), and the eviction of the tokens that received least (evict).

With `own` false, run computes each of them from elementary torch operations in 32 bits; with `own` true it calls the
library.  exact computes them once more in 64 bits, sequence by sequence.

Head layouts are those of the decoders in paper_2601_19404_amd/synth.py (tiny fp32, 1.5B- and 7B-shaped) and a generic one
of 64 channels; prefix, suffix and batch sizes those of its workloads (64 groups of 8, trajectories of 2048 and 4096 tokens
cut in the last 5 - 10 %), batches of a few sequences and caches of up to some 30000 tokens.

Pages: [2 (keys, values), KV heads, ...], keys [page_tokens, channels], values [page_tokens / 8, channels, 8].
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# name: query heads, KV heads, channels of a head, element type, tokens of a page
LAYOUTS = {"tiny": (4, 2, 32, "f32", 16), "1.5b": (12, 2, 128, "bf16", 64), "7b": (28, 4, 128, "bf16", 64),
           "h64": (16, 4, 64, "bf16", 32), "1.5b_f32": (12, 2, 128, "f32", 64)}


def _case(name, kind, layout, seqs, len_lo, len_hi, new_lo=1, new_hi=1, window=0, sinks=0, lse=False, budget=0,
          recent=0, shape_seed=1):
    """seqs sequences whose caches hold len_lo..len_hi tokens, the last new_lo..new_hi of which are the call's rows."""
    c = dict(kind=kind, layout=layout, seqs=seqs, len_lo=len_lo, len_hi=len_hi, new_lo=new_lo, new_hi=new_hi,
             window=window, sinks=sinks, lse=lse, budget=budget, recent=recent, shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one question's next token: latency
        _case("attn_decode_1.5b_1", "attn", "1.5b", 1, 2176, 2176),
        # a decode step of a large batch with caches of their own, long trajectories: memory
        _case("attn_decode_7b_128", "attn", "7b", 128, 4000, 4505),
        # a decode step of the headline batch under a window with sinks
        _case("attn_decode_1.5b_512_window", "attn", "1.5b", 512, 1900, 2250, window=512, sinks=4),
        # prefill of whole trajectories, the statistics kept for the scores: matrix units
        _case("attn_prefill_7b_4", "attn", "7b", 4, 4352, 4352, 4352, 4352, lse=True),
        # scoring ragged suffixes against long prefixes under a window with sinks
        _case("attn_suffix_1.5b_64_window", "attn", "1.5b", 64, 1900, 2250, 103, 204, window=1024, sinks=4),
        # the fp32 decoder of the tests: a few rows, latency
        _case("attn_tiny_8", "attn", "tiny", 8, 40, 80, 8, 16, lse=True),
        # every decode step of a batch that will evict adds its weights
        _case("score_decode_1.5b_512", "score", "1.5b", 512, 1900, 2250),
        # weights that the tokens of whole trajectories give each other
        _case("score_prefill_7b_4", "score", "7b", 4, 4352, 4352, 4352, 4352),
        # a batch of trajectories cut to a budget
        _case("evict_1.5b_64", "evict", "1.5b", 64, 1900, 2250, sinks=4, budget=1024, recent=256),
        # two long caches cut to an eighth
        _case("evict_7b_2_long", "evict", "7b", 2, 15000, 16384, sinks=4, budget=2048, recent=512),
        # a decode step's keys and values
        _case("append_decode_1.5b_512", "append", "1.5b", 512, 1900, 2250),
        # a prefill's keys and values
        _case("append_prefill_7b_4", "append", "7b", 4, 4352, 4352, 4352, 4352),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = max((work(c) for c in listed()), key=lambda w: w["flops"])["flops"]
    while True:
        kind = rng.choice(["attn", "attn", "attn", "attn", "score", "score", "evict", "evict", "append", "append"])
        layout = rng.choice(["tiny", "1.5b", "1.5b", "7b", "7b", "h64", "1.5b_f32"])
        seqs = log(1, 512)
        hi = log(24, 400) if layout == "tiny" else log(8, 32000 if kind != "append" else 8000)
        lo = max(1, int(hi * rng.uniform(0.4, 1.0)))
        new_hi = rng.choice([1, 1, log(2, 8), log(2, hi), hi]) if kind != "evict" else 1
        new_hi = min(new_hi, hi)
        new_lo = max(1, int(new_hi * rng.uniform(0.3, 1.0)))
        windowed = kind in ("attn", "score") and rng.random() < 0.5
        window = log(1, 2 * hi) if windowed else 0
        sinks = rng.choice([0, 1, 4, 7, 64, 100]) if windowed or kind == "evict" else 0
        budget = recent = 0
        if kind == "evict":
            budget = max(sinks + 1, int(hi * rng.uniform(0.1, 1.0)))
            recent = rng.randint(0, budget - sinks)
        case = _case(None, kind, layout, seqs, lo, hi, new_lo, new_hi, window, sinks, kind == "attn" and rng.random() < 0.5,
                     budget, recent, rng.randrange(1 << 20))
        w, (Hq, Hkv, dh, dt, pt) = work(case), LAYOUTS[layout]
        plain = 4.0 * seqs * max(Hq * new_hi * hi if kind in ("attn", "score") else 0, 2 * Hkv * hi * dh)
        if w["flops"] <= most * (0.1 if dt == "f32" else 1) and w["bytes"] <= 1.2e9 and plain <= 8.6e9:
            return case


# ---------------------------------------------------------------------------------------------
def _shapes(case):
    """Tokens in the cache and new rows of every sequence."""
    r = np.random.Generator(np.random.PCG64(case["shape_seed"]))
    n = case["seqs"]
    ln = r.integers(case["len_lo"], case["len_hi"] + 1, size=n)
    new = np.minimum(r.integers(case["new_lo"], case["new_hi"] + 1, size=n), ln)
    return ln.astype(np.int64), new.astype(np.int64)


def _cache(g, n_seqs, tokens, Hkv, dh, dt, pt, fill):
    """A pool with room for `tokens` of every sequence and a few pages more, and the sequences' pages in random order."""
    per = -(-tokens // pt)
    n_pages = n_seqs * per + 3
    shape = (n_pages, 2 * Hkv * pt * dh)
    pool = (torch.randn(shape, device="cuda", generator=g, dtype=dt) if fill
            else torch.zeros(shape, device="cuda", dtype=dt))
    table = torch.randperm(n_pages, device="cuda", generator=g)[: n_seqs * per].to(torch.int32).view(n_seqs, per)
    return dict(pool=pool, table=table.contiguous(), Hkv=Hkv, dh=dh, pt=pt)


def prepare(case, seed):
    Hq, Hkv, dh, dt, pt = LAYOUTS[case["layout"]]
    dt = torch.float32 if dt == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ln, new = _shapes(case)
    n, longest, most_new = case["seqs"], int(ln.max()), int(new.max())
    st = dict(case=case, longest=longest, most_new=most_new, Hq=Hq)
    c = st["cache"] = _cache(g, n, longest, Hkv, dh, dt, pt, case["kind"] != "append")
    c["len"] = torch.from_numpy(ln.astype(np.int32)).cuda()
    st["cu"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
    rows = int(new.sum())
    if case["kind"] == "append":          # keys and values as the QKV projection leaves them: columns of one wide array
        wide = torch.randn(rows, (Hq + 2 * Hkv) * dh, device="cuda", generator=g, dtype=dt)
        st["k"], st["v"] = wide[:, Hq * dh: (Hq + Hkv) * dh], wide[:, (Hq + Hkv) * dh:]
    if case["kind"] in ("attn", "score"):  # query . key with a spread of 2: some tokens matter, most do not
        st["q"] = (2.0 * torch.randn(rows, Hq * dh, device="cuda", generator=g)).to(dt)
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros(rows, Hq, device="cuda")
    if case["kind"] == "score":
        st["lse"] = math.log(max(1, longest)) + 2.0 + 0.3 * torch.randn(rows, Hq, device="cuda", generator=g)
    if case["kind"] in ("score", "evict"):  # weights of earlier steps: a few tokens hold most of them; many equal ones
        s = torch.exp(1.5 * torch.randn(n, Hkv, longest, device="cuda", generator=g))
        s[..., ::3] = torch.round(s[..., ::3] * 8) / 8
        st["score"] = s
        st["score_out"] = torch.zeros_like(s)
    if case["kind"] == "evict":
        b = case["budget"]
        st["to"] = _cache(g, n, b, Hkv, dh, dt, pt, False)
        st["to"]["len"] = torch.zeros(n, dtype=torch.int32, device="cuda")
        st["kept"] = torch.zeros(n, Hkv, b, dtype=torch.int32, device="cuda")
        st["score_out"] = torch.zeros(n, Hkv, b, device="cuda")
    if own:
        from paper_2601_19404_amd import binding as rpo
        for key in ("cache", "to"):
            if key in st:
                x = st[key]
                st["paged_" + key] = rpo.PagedKV(x["pool"], x["table"], x["len"], x["pt"], x["Hkv"], x["dh"])
        if case["kind"] in ("attn", "score"):
            size = rpo.rpo_attn_paged_ws_bytes if case["kind"] == "attn" else rpo.rpo_kv_score_ws_bytes
            need = size(st["paged_cache"], rows, most_new, longest, Hq, case["window"], case["sinks"])
            st["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return st


def run(st):
    return (_own if own else _plain)[st["case"]["kind"]](st)


# ---- the library's calls ------------------------------------------------------------------------
def _own_append(st):
    from paper_2601_19404_amd import binding as rpo
    rpo.rpo_kv_append(st["paged_cache"], st["k"], st["v"], st["cu"], st["most_new"])
    return dict(pool=st["cache"]["pool"])


def _own_attn(st):
    from paper_2601_19404_amd import binding as rpo
    c = st["case"]
    lse = st["lse"] if c["lse"] else None
    rpo.rpo_attn_paged(st["paged_cache"], st["q"], st["cu"], st["most_new"], st["out"], window=c["window"],
                       n_sinks=c["sinks"], lse_out_dev=lse, ws_dev=st["ws"], max_len=st["longest"])
    return dict(out=st["out"], lse=lse) if c["lse"] else dict(out=st["out"])


def _own_score(st):
    from paper_2601_19404_amd import binding as rpo
    c = st["case"]
    rpo.rpo_kv_score(st["paged_cache"], st["q"], st["cu"], st["most_new"], st["lse"], st["score"], st["score_out"],
                     window=c["window"], n_sinks=c["sinks"], ws_dev=st["ws"], max_len=st["longest"])
    return dict(score=st["score_out"])


def _own_evict(st):
    from paper_2601_19404_amd import binding as rpo
    c = st["case"]
    rpo.rpo_kv_evict(st["paged_cache"], st["score"], c["budget"], c["sinks"], c["recent"], st["paged_to"],
                     st["to"]["len"], st["kept"], st["score_out"])
    return dict(pool=st["to"]["pool"], length=st["to"]["len"], kept=st["kept"], score=st["score_out"])


_own = {"append": _own_append, "attn": _own_attn, "score": _own_score, "evict": _own_evict}


# ---- the plain forms ----------------------------------------------------------------------------
def _views(c):
    """Keys [pages, KV heads, tokens, channels] and values [pages, KV heads, tokens / 8, channels, 8] of a pool."""
    p = c["pool"].view(-1, 2, c["Hkv"], c["pt"] * c["dh"])
    return (p[:, 0].view(-1, c["Hkv"], c["pt"], c["dh"]), p[:, 1].view(-1, c["Hkv"], c["pt"] // 8, c["dh"], 8))


def _row_slots(st):
    """Row of every (sequence, new token), its slot in the cache and whether there is such a row."""
    c, cu = st["cache"], st["cu"].long()
    n = cu[1:] - cu[:-1]
    i = torch.arange(st["most_new"], device="cuda")[None]
    there = i < n[:, None]
    return (cu[:-1, None] + i).clamp_(max=int(st["q"].shape[0] if "q" in st else st["k"].shape[0]) - 1), \
        (c["len"].long() - n)[:, None] + i, there


def _plain_append(st):
    c = st["cache"]
    K, V = _views(c)
    rows, slot, there = _row_slots(st)
    page = c["table"].long().gather(1, slot // c["pt"])[there]
    rows, at = rows[there], slot[there] % c["pt"]
    K[page, :, at] = st["k"][rows].view(-1, c["Hkv"], c["dh"])
    V[page, :, at // 8, :, at % 8] = st["v"][rows].view(-1, c["Hkv"], c["dh"])
    return dict(pool=c["pool"])


def _plain_scores(st):
    """scale q . k in 32 bits, [sequences, KV heads, heads of one, new rows, tokens], -inf where a row does not see."""
    c, case, L = st["cache"], st["case"], st["longest"]
    K = _views(c)[0]
    S, hpk = c["table"].shape[0], st["Hq"] // c["Hkv"]
    rows, slot, there = _row_slots(st)
    k = K[c["table"].long()].transpose(1, 2).reshape(S, c["Hkv"], -1, c["dh"])[:, :, :L].float()
    q = st["q"].view(-1, c["Hkv"], hpk, c["dh"])[rows].permute(0, 2, 3, 1, 4).float()   # [S, Hkv, hpk, new, dh]
    s = torch.matmul(q.reshape(S, c["Hkv"], -1, c["dh"]), k.transpose(2, 3)).view(S, c["Hkv"], hpk, -1, L)
    s *= 1.0 / math.sqrt(c["dh"])
    j = torch.arange(L, device="cuda")
    seen = (j <= slot[..., None]) & there[..., None]
    if case["window"]:
        seen &= (j > slot[..., None] - case["window"]) | (j < case["sinks"])
    return s.masked_fill_(~seen[:, None, None], -math.inf), rows, there


def _plain_attn(st):
    c, case, L = st["cache"], st["case"], st["longest"]
    S, Hkv, dh = c["table"].shape[0], c["Hkv"], c["dh"]
    s, rows, there = _plain_scores(st)
    top = s.amax(dim=-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = s.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    v = _views(c)[1][c["table"].long()].permute(0, 2, 1, 3, 5, 4).reshape(S, Hkv, -1, dh)[:, :, :L].float()
    o = torch.matmul(p.view(S, Hkv, -1, L), v).view(*p.shape[:-1], dh) / torch.where(total == 0, 1.0, total)
    st["out"][rows[there]] = o.permute(0, 3, 1, 2, 4).reshape(S, -1, st["Hq"] * dh)[there].to(st["out"].dtype)
    if not case["lse"]:
        return dict(out=st["out"])
    st["lse"][rows[there]] = (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(S, -1, st["Hq"])[there]
    return dict(out=st["out"], lse=st["lse"])


def _plain_score(st):
    c = st["cache"]
    s, rows, there = _plain_scores(st)
    lse = st["lse"].view(-1, c["Hkv"], st["Hq"] // c["Hkv"])[rows].permute(0, 2, 3, 1)
    p = s.sub_(lse[..., None]).exp_()
    held = torch.arange(st["longest"], device="cuda") < c["len"][:, None]
    st["score_out"].copy_(torch.where(held[:, None], st["score"] + p.sum(dim=(2, 3)), st["score_out"]))
    return dict(score=st["score_out"])


def _plain_evict(st):
    c, to, case, L = st["cache"], st["to"], st["case"], st["longest"]
    b, Hkv, dh = case["budget"], c["Hkv"], c["dh"]
    ln = c["len"].long()
    j = torch.arange(L, device="cuda")
    always = (j < case["sinks"]) | (j >= ln[:, None] - case["recent"]) | (ln[:, None] <= b)
    rank = torch.where(always[:, None], math.inf, st["score"])
    rank = torch.where((j < ln[:, None])[:, None], rank, -math.inf)
    first = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :b]
    if first.shape[-1] < b:
        first = torch.cat([first, first.new_full((*first.shape[:-1], b - first.shape[-1]), L)], dim=-1)
    held = torch.minimum(ln, ln.new_tensor(b))
    live = (torch.arange(b, device="cuda") < held[:, None])[:, None].expand_as(first)
    kept = torch.where(live, first, L).sort(dim=-1).values
    st["kept"].copy_(torch.where(live, kept, -1))
    old = kept.clamp(max=L - 1)
    st["score_out"].copy_(torch.where(live, st["score"].gather(2, old), 0.0))
    to["len"].copy_(held)
    s, h, i = live.nonzero(as_tuple=True)
    old = old[s, h, i]
    page, new_page = c["table"].long()[s, old // c["pt"]], to["table"].long()[s, i // to["pt"]]
    (K, V), (K2, V2) = _views(c), _views(to)
    K2[new_page, h, i % to["pt"]] = K[page, h, old % c["pt"]]
    V2[new_page, h, i % to["pt"] // 8, :, i % 8] = V[page, h, old % c["pt"] // 8, :, old % 8]
    return dict(pool=to["pool"], length=to["len"], kept=st["kept"], score=st["score_out"])


_plain = {"append": _plain_append, "attn": _plain_attn, "score": _plain_score, "evict": _plain_evict}


# ---------------------------------------------------------------------------------------------
def _token_offsets(c, s, slots):
    """Element offsets in the pool, [KV heads, slots, channels], of the keys and of the values of a sequence's slots."""
    slots = torch.as_tensor(slots, device="cuda", dtype=torch.int64)
    page, at = c["table"][s].long()[slots // c["pt"]], slots % c["pt"]
    block = c["pt"] * c["dh"]
    d = torch.arange(c["dh"], device="cuda")
    h = torch.arange(c["Hkv"], device="cuda")[:, None, None]
    base = (page * 2 * c["Hkv"] * block)[None, :, None]
    return (base + h * block + (at * c["dh"])[None, :, None] + d,
            base + (c["Hkv"] + h) * block + ((at // 8) * c["dh"] * 8)[None, :, None] + d * 8 + (at % 8)[None, :, None])


def exact(case, seed):
    """What run returns, in 64 bits, one sequence and KV head after the other."""
    st = prepare(case, seed)
    ln, new = _shapes(case)
    c, kind = st["cache"], case["kind"]
    flat, dh, hpk = c["pool"].view(-1), c["dh"], st["Hq"] // c["Hkv"]
    first = np.concatenate([[0], np.cumsum(new)])
    if kind == "append":
        for s in range(case["seqs"]):
            a, b = int(first[s]), int(first[s + 1])
            ko, vo = _token_offsets(c, s, np.arange(ln[s] - new[s], ln[s]))
            flat[ko.transpose(0, 1).reshape(b - a, -1)] = st["k"][a:b]
            flat[vo.transpose(0, 1).reshape(b - a, -1)] = st["v"][a:b]
        return dict(pool=c["pool"].double())
    if kind == "evict":
        to, b = st["to"], case["budget"]
        score = st["score"].cpu().numpy()
        kept = np.full((case["seqs"], c["Hkv"], b), -1, dtype=np.int64)
        weights = np.zeros(kept.shape)
        for s in range(case["seqs"]):
            held = int(min(b, ln[s]))
            for h in range(c["Hkv"]):
                slots = np.arange(ln[s])
                if ln[s] > b:
                    mid = slots[case["sinks"]: ln[s] - case["recent"]]
                    best = mid[np.lexsort((mid, -score[s, h, mid]))[: b - case["sinks"] - case["recent"]]]
                    slots = np.sort(np.concatenate([slots[: case["sinks"]], best, slots[ln[s] - case["recent"]:]]))
                kept[s, h, :held], weights[s, h, :held] = slots, score[s, h, slots]
                (ko, vo), (kn, vn) = _token_offsets(c, s, slots), _token_offsets(to, s, np.arange(held))
                target = to["pool"].view(-1)
                target[kn[h]] = flat[ko[h]]
                target[vn[h]] = flat[vo[h]]
        return dict(pool=to["pool"].double(), length=torch.from_numpy(np.minimum(ln, b)).to(torch.int32),
                    kept=torch.from_numpy(kept).to(torch.int32), score=torch.from_numpy(weights))
    out = torch.zeros(*st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(*st["lse"].shape, dtype=torch.float64, device="cuda")
    score = st["score"].double() if kind == "score" else None
    for s in range(case["seqs"]):
        a, b, T = int(first[s]), int(first[s + 1]), int(ln[s])
        ko, vo = _token_offsets(c, s, np.arange(T))
        at = torch.arange(T - (b - a), T, device="cuda")[:, None]
        j = torch.arange(T, device="cuda")[None]
        hidden = j > at
        if case["window"]:
            hidden |= (at - j >= case["window"]) & (j >= case["sinks"])
        for h in range(st["Hq"]):
            g = h // hpk
            z = st["q"][a:b, h * dh:(h + 1) * dh].double() @ flat[ko[g]].double().t() / math.sqrt(dh)
            if kind == "attn":
                lse[a:b, h] = torch.logsumexp(z.masked_fill(hidden, -math.inf), dim=1)
                out[a:b, h * dh:(h + 1) * dh] = torch.softmax(z.masked_fill(hidden, -math.inf), dim=1) @ flat[vo[g]].double()
            else:
                score[s, g, :T] += torch.exp(z - st["lse"][a:b, h, None].double()).masked_fill(hidden, 0.0).sum(dim=0)
    if kind == "attn":
        return dict(out=out, lse=lse) if case["lse"] else dict(out=out)
    held = torch.arange(st["longest"], device="cuda") < c["len"][:, None]
    return dict(score=torch.where(held[:, None], score, 0.0))


# ---------------------------------------------------------------------------------------------
def work(case):
    Hq, Hkv, dh, dt, pt = LAYOUTS[case["layout"]]
    es = 4 if dt == "f32" else 2
    ln, new = (x.astype(np.float64) for x in _shapes(case))
    token = 2.0 * Hkv * dh * es                              # one token's keys and values
    if case["kind"] == "append":
        return dict(bytes=float(new.sum()) * 2 * token, flops=0.0)
    if case["kind"] == "evict":
        held = np.minimum(ln, case["budget"])
        return dict(bytes=float(ln.sum() * Hkv * 4 + held.sum() * (2 * token + Hkv * 8)), flops=float(ln.sum() * Hkv))
    pairs = slots = 0.0
    for T, n in zip(ln, new):                                # rows at slots T - n .. T - 1
        t = np.arange(T - n, T)
        if not case["window"]:
            pairs, slots = pairs + float((t + 1).sum()), slots + T
            continue
        lo = np.maximum(0, t - case["window"] + 1)           # first slot of a row's window
        pairs += float((t + 1 - lo + np.minimum(lo, case["sinks"])).sum())
        slots += T - lo[0] + min(lo[0], case["sinks"])
    rows = float(new.sum()) * Hq
    if case["kind"] == "attn":
        return dict(bytes=slots * token + rows * (2 * dh * es + (4 if case["lse"] else 0)), flops=4.0 * dh * pairs * Hq)
    return dict(bytes=slots * token / 2 + rows * (dh * es + 4) + float(ln.sum()) * Hkv * 8, flops=2.0 * dh * pairs * Hq)
