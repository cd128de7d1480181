"""What the paged attention's gradient refuses before anything is launched (CPU: addresses are never read, and the context is a
block of zeros behind its first field, the shape)."""
import ctypes as C

import pytest

from paper_2605_07230_b200 import binding as cb

N_TOK, N_KV, HQ, HKV, D = 10, 40, 4, 2, 64
NAMES = ("q", "q_begin", "kv_len", "out", "lse", "d_out", "scratch", "dq", "dk", "dv", "k_begin", "k_pages", "v_pages", "table")
AT = {name: 0x10000000 * (i + 1) for i, name in enumerate(NAMES)}


def call(dtype=cb.BF16, ctx_shape=None, **kw):
    a = dict(AT, n_req=2, n_tok=N_TOK, n_kv=N_KV, max_q=8, max_kv=30, window=0, sinks=0, scale=0.1, page_stride=16 * HKV * D, n_pages=6, page=16,
             table_stride=4, width=0, **{s: HQ * D for s in ("q_stride", "dq_stride")}, **{s: HKV * D for s in ("dk_stride", "dv_stride")})
    a.update(kw)
    block = C.create_string_buffer(1 << 16)
    shape = cb.Shape(*(ctx_shape or (dtype, 1, 1, 64, 64, HQ, HKV, D, 64, 0)))
    C.memmove(block, C.byref(shape), C.sizeof(shape))
    cache = cb.PagedCacheStruct(a["k_pages"], a["v_pages"], a["page_stride"], a["n_pages"], a["page"], a["table"], a["table_stride"], a["width"])
    return cb.lib().cascade_paged_attn_grad(
        None if a.get("ctx", 1) is None else block, None if a.get("cache", 1) is None else C.byref(cache), a["n_req"], a["n_tok"], a["q"],
        a["q_stride"], a["q_begin"], a["kv_len"], a["max_q"], a["max_kv"], a["window"], a["sinks"], a["scale"], a["out"], a["lse"], a["d_out"],
        a["scratch"], a["dq"], a["dq_stride"], a["dk"], a["dk_stride"], a["dv"], a["dv_stride"], a["n_kv"], a["k_begin"], None)


NAN, INF = float("nan"), float("inf")
ROW, KV_ROW = HQ * D * 2, HKV * D * 2           # bytes


@pytest.mark.parametrize("kw", [{name: None} for name in NAMES + ("ctx", "cache") if name != "k_begin"])
def test_null_pointers(kw):
    assert call(**kw) == cb.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(n_req=0), dict(n_tok=0), dict(n_kv=0), dict(max_q=0), dict(max_kv=-1), dict(window=-1), dict(sinks=-1),
                                dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(table_stride=0), dict(width=5),
                                dict(width=-1), dict(n_pages=0), dict(page=0), dict(page_stride=16 * HKV * D - 8),
                                dict(q_stride=HQ * D - 8), dict(dq_stride=HQ * D - 8), dict(dk_stride=HKV * D - 8), dict(dv_stride=0),
                                dict(q_stride=HQ * D + 4), dict(dk_stride=HKV * D + 1), dict(dv_stride=2**41), dict(dq_stride=2**41)])
def test_sizes_and_strides(kw):
    assert call(**kw) == cb.ERR_INVALID_ARG


@pytest.mark.parametrize("name", ["q", "out", "d_out", "scratch", "dq", "dk", "dv", "k_pages", "v_pages"])
def test_alignment_to_16_bytes(name):
    assert call(**{name: AT[name] + 8}) == cb.ERR_INVALID_ARG


@pytest.mark.parametrize("name", ["q_begin", "kv_len", "lse", "k_begin", "table"])
def test_alignment_to_4_bytes(name):
    assert call(**{name: AT[name] + 2}) == cb.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(dq=AT["q"]), dict(dq=AT["q"] + (N_TOK - 1) * ROW), dict(dk=AT["dv"]), dict(dv=AT["dk"] + (N_KV - 1) * KV_ROW),
                                dict(dq=AT["out"]), dict(scratch=AT["d_out"]), dict(dk=AT["lse"]), dict(dk=AT["k_pages"]),
                                dict(dv=AT["v_pages"] + 5 * 16 * KV_ROW), dict(scratch=AT["dq"]), dict(dq=AT["d_out"]),
                                # one stacked gradient whose parts overlap by one element
                                dict(dq_stride=512, dk_stride=512, dv_stride=512, dk=AT["dq"] + ROW - 16),
                                dict(dq_stride=512, dk_stride=512, dv_stride=512, dk=AT["dq"] + 1024 - KV_ROW + 16),
                                dict(dq=AT["q_begin"]), dict(dk=AT["kv_len"] - KV_ROW), dict(scratch=AT["k_begin"]),
                                dict(dv=AT["table"] + 16),
                                # rows farther apart than 64 bits count
                                dict(n_kv=2**31 - 1, dk_stride=2**40)])
def test_overlaps(kw):
    assert call(**kw) == cb.ERR_INVALID_ARG


def test_sizes_past_32_bits():
    assert call(max_kv=2**31 - 65535) == cb.ERR_UNSUPPORTED_SHAPE
    assert call(n_req=cb.MAX_REQUESTS + 1) == cb.ERR_UNSUPPORTED_SHAPE
    assert call(ctx_shape=(cb.BF16, 1, 1, 64, 64, 258, 2, 64, 64, 0), q_stride=258 * 64, dq_stride=258 * 64) == cb.ERR_UNSUPPORTED_SHAPE
    assert call(page=12) == cb.ERR_UNSUPPORTED_SHAPE
