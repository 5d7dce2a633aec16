"""What the paged-cache entry points refuse on the host, before anything is enqueued (no GPU needed): every call here has
one wrong argument and must come back with the error code, and with nothing launched (there is no device to launch on)."""
import ctypes as C

import pytest

from paper_2601_19404_amd import binding as b

P = 1 << 20      # an aligned address that is never looked at


def _kv(**kw):
    d = dict(pool_dev=P, table_dev=P, len_dev=P, page_stride=2 * 2 * 64 * 128, n_pages=10, n_seqs=3, table_stride=4,
             page_tokens=64, n_kv_heads=2, head_dim=128, dtype=b.RPO_BF16)
    d.update(kw)
    return b.PagedKvDesc(*[d[n] for n, _ in b.PagedKvDesc._fields_])


BAD_CACHES = [dict(pool_dev=None), dict(table_dev=None), dict(len_dev=None), dict(dtype=2), dict(n_seqs=-1),
              dict(n_seqs=65536), dict(n_pages=0), dict(table_stride=0), dict(n_kv_heads=0), dict(head_dim=127),
              dict(head_dim=258), dict(head_dim=0), dict(page_tokens=8), dict(page_tokens=48),
              dict(table_stride=1 << 25), dict(page_stride=2 * 2 * 64 * 128 - 8), dict(page_stride=2 * 2 * 64 * 128 + 4),
              dict(pool_dev=P + 8)]


def _append(kv, **kw):
    a = dict(k=P, k_stride=256, v=P, v_stride=256, cu=P, n_rows=5, max_new=2)
    a.update(kw)
    return b.lib().rpo_kv_append(kv, a["k"], a["k_stride"], a["v"], a["v_stride"], a["cu"], a["n_rows"], a["max_new"], None)


ATTN = dict(q=P, q_stride=1536, cu=P, n_rows=5, max_new=2, max_len=200, Hq=12, scale=0.1, window=0, sinks=0, out=P,
            out_stride=1536, lse=None, ws=None, ws_bytes=0)


def _attn(kv, **kw):
    a = dict(ATTN, **kw)
    return b.lib().rpo_attn_paged(kv, a["q"], a["q_stride"], a["cu"], a["n_rows"], a["max_new"], a["max_len"], a["Hq"],
                                  a["scale"], a["window"], a["sinks"], a["out"], a["out_stride"], a["lse"], a["ws"],
                                  a["ws_bytes"], None)


def _score(kv, **kw):
    a = dict(ATTN, lse=P, score_in=None, score_out=P, score_stride=256)
    a.update(kw)
    return b.lib().rpo_kv_score(kv, a["q"], a["q_stride"], a["cu"], a["n_rows"], a["max_new"], a["max_len"], a["Hq"],
                                a["scale"], a["window"], a["sinks"], a["lse"], a["score_in"], a["score_out"],
                                a["score_stride"], a["ws"], a["ws_bytes"], None)


def _evict(kv, dst=None, **kw):
    a = dict(score=P, score_stride=256, budget=100, sinks=4, recent=10, len_out=P, score_out=None, score_out_stride=0, kept=P)
    a.update(kw)
    dst = _kv(pool_dev=2 * P, table_dev=3 * P, len_dev=None) if dst is None else dst
    return b.lib().rpo_kv_evict(kv, a["score"], a["score_stride"], a["budget"], a["sinks"], a["recent"], dst, a["len_out"],
                                a["score_out"], a["score_out_stride"], a["kept"], None)


@pytest.mark.parametrize("call", [_append, _attn, _score, _evict])
@pytest.mark.parametrize("wrong", BAD_CACHES, ids=lambda d: "-".join(f"{k}{v}" for k, v in d.items()))
def test_bad_caches(call, wrong):
    assert call(_kv(**wrong)) == b.RPO_EINVAL
    assert call(None) == b.RPO_EINVAL and "NULL cache" in b.rpo_last_error()


@pytest.mark.parametrize("wrong", [dict(k=None), dict(v=None), dict(cu=None), dict(n_rows=-1), dict(max_new=-1),
                                   dict(max_new=6), dict(k_stride=255), dict(v_stride=255), dict(k=P + 1),
                                   dict(n_rows=(1 << 30) + 1)])
def test_append_refuses(wrong):
    assert _append(_kv(), **wrong) == b.RPO_EINVAL and "rpo_kv_append" in b.rpo_last_error()


ATTN_WRONG = [dict(q=None), dict(cu=None), dict(q_stride=1535), dict(n_rows=-1), dict(max_new=-1), dict(max_new=6),
              dict(max_len=-1), dict(Hq=0), dict(Hq=13), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
              dict(scale=float("inf")), dict(window=-1), dict(sinks=-1), dict(ws=P), dict(ws_bytes=64),
              dict(ws=P + 8, ws_bytes=1 << 30), dict(q=P + 1), dict(n_rows=1 << 30, max_new=1 << 30)]


@pytest.mark.parametrize("wrong", ATTN_WRONG + [dict(out=None), dict(out_stride=1535), dict(out=P + 1)])
def test_attention_refuses(wrong):
    assert _attn(_kv(), **wrong) == b.RPO_EINVAL and "rpo_attn_paged" in b.rpo_last_error()


@pytest.mark.parametrize("wrong", ATTN_WRONG + [dict(lse=None), dict(score_out=None), dict(score_stride=0)])
def test_score_refuses(wrong):
    assert _score(_kv(), **wrong) == b.RPO_EINVAL and "rpo_kv_score" in b.rpo_last_error()


@pytest.mark.parametrize("wrong", [dict(score=None), dict(len_out=None), dict(kept=None), dict(budget=0), dict(budget=13),
                                   dict(budget=257), dict(sinks=-1), dict(recent=-1), dict(score_stride=0),
                                   dict(score_out=2 * P, score_out_stride=99), dict(score_out=P, score_out_stride=256),
                                   dict(sinks=2**31 - 1, recent=2**31 - 1)])
def test_evict_refuses(wrong):
    assert _evict(_kv(), **wrong) == b.RPO_EINVAL and "rpo_kv_evict" in b.rpo_last_error()


@pytest.mark.parametrize("other", [dict(n_seqs=2), dict(n_kv_heads=1), dict(head_dim=64), dict(dtype=b.RPO_F32),
                                   dict(pool_dev=None), dict(page_tokens=24)])
def test_evict_refuses_another_layout_behind(other):
    assert _evict(_kv(), _kv(**dict(dict(pool_dev=2 * P, len_dev=None), **other))) == b.RPO_EINVAL
    assert _evict(_kv(), _kv()) == b.RPO_EINVAL and "must not be src's" in b.rpo_last_error()


def test_workspace_sizes_run_on_the_host_and_too_small_ones_are_refused():
    L, kv = b.lib(), _kv(n_seqs=1, table_stride=100)
    for size, call in ((L.rpo_attn_paged_ws_bytes, _attn), (L.rpo_kv_score_ws_bytes, _score)):
        assert size(None, 1, 1, 4000, 12, 0, 0) == 0 and size(kv, 1, 2, 4000, 12, 0, 0) == 0     # refused: 0
        need = size(kv, 1, 1, 4000, 12, 0, 0)
        assert need % 4 == 0
        if need:
            assert call(kv, n_rows=1, max_new=1, max_len=4000, ws=P, ws_bytes=need - 1) == b.RPO_ENOMEM
    assert L.rpo_batch_kv(None, 0, C.byref(_kv())) == b.RPO_EINVAL


def test_no_sequences_and_no_rows_are_fine_without_a_device():
    empty = _kv(n_seqs=0)
    assert _append(empty) == b.RPO_OK and _attn(empty) == b.RPO_OK and _score(empty) == b.RPO_OK
    assert _evict(empty, _kv(n_seqs=0, pool_dev=2 * P)) == b.RPO_OK
    assert _append(_kv(), n_rows=0, max_new=0, k=None, v=None) == b.RPO_OK
    assert _attn(_kv(), n_rows=0, max_new=0, q=None, out=None) == b.RPO_OK


def test_binding_refuses_host_tensors():
    import torch
    pool = torch.zeros(4, 2 * 2 * 16 * 32)
    with pytest.raises(ValueError):
        b.PagedKV(pool, torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 16, 2, 32)


def test_binding_refuses_numbers_that_32_bits_do_not_hold():
    """2^32 would reach the library as 0: no window, an empty cache."""
    import types
    kv = types.SimpleNamespace(ref=C.byref(_kv(n_seqs=1, table_stride=100)))
    for size in (b.rpo_attn_paged_ws_bytes, b.rpo_kv_score_ws_bytes):
        assert size(kv, 200, 200, 4000, 12) > 0 and size(kv, 200, 200, 4000, 12, 2 ** 31 - 1, 2 ** 31 - 1) > 0
        for wrong in ((2 ** 32 + 200, 200, 4000, 12), (200, 200, 2 ** 32 + 4000, 12), (200, 200, 4000, 2 ** 32 + 12),
                      (200, 200, 4000, 12, 2 ** 32), (200, 200, 4000, 12, 4, 2 ** 31), (200, -2 ** 32 + 200, 4000, 12)):
            with pytest.raises(ValueError):
                size(kv, *wrong)
        assert size(kv, 200, 200, 4000, 12, -1) == 0               # below 0: the library's own refusal


def test_what_one_launch_does_not_hold_is_refused_before_anything_is_enqueued():
    many = dict(n_seqs=65535, n_kv_heads=1024, head_dim=32, page_stride=2 * 1024 * 64 * 32)
    wide = dict(Hq=1024, q_stride=1024 * 32, out_stride=1024 * 32)
    assert _attn(_kv(**many), **wide) == b.RPO_EINVAL and "one launch" in b.rpo_last_error()
    assert _score(_kv(**many), **wide) == b.RPO_EINVAL and "one launch" in b.rpo_last_error()
    long = dict(table_stride=1 << 24)                                  # 2^30 slots
    assert _score(_kv(**long, n_seqs=8), max_len=1 << 30) == b.RPO_EINVAL and "one launch" in b.rpo_last_error()
    odd = dict(long, head_dim=96, page_stride=2 * 2 * 64 * 96)          # the generic kernel: 32 slots a workgroup
    assert _score(_kv(**odd), max_len=1 << 30) == b.RPO_EINVAL and "one launch" in b.rpo_last_error()
    to = _kv(pool_dev=2 * P, len_dev=None, **long)
    assert _evict(_kv(**long), to, budget=1 << 30) == b.RPO_EINVAL and "budget" in b.rpo_last_error()


def test_a_workspace_that_is_too_small_is_refused_by_every_call_that_splits():
    L, kv = b.lib(), _kv(n_seqs=1, table_stride=100)
    for size, call, new in ((L.rpo_attn_paged_ws_bytes, _attn, 1), (L.rpo_attn_paged_ws_bytes, _attn, 200),
                            (L.rpo_kv_score_ws_bytes, _score, 200)):
        need = size(kv, new, new, 4000, 12, 0, 0)
        assert need > 0
        assert call(kv, n_rows=new, max_new=new, max_len=4000, ws=P, ws_bytes=need - 1) == b.RPO_ENOMEM
        assert "%d needed" % need in b.rpo_last_error()
