"""Refusals of the paged-cache and rotary calls: validated on the host before any launch, so no GPU is needed."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2511_12201_amd import binding as ob

FAKE = 0x10000            # non-null, 256-byte aligned; never dereferenced: validation fails first
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return ob.load_library()


def _chunk(**kw):
    d = ob.ChunkDesc()
    d.batch, d.n_q_heads, d.n_kv_heads, d.head_dim, d.n_new, d.causal, d.dtype = 2, 4, 2, 64, 5, 1, ob.OMNI_BF16
    d.softmax_scale = 0.125
    d.q_stride = (C.c_int64 * 3)(4 * 5 * 64, 5 * 64, 64)
    d.kv_stride = (C.c_int64 * 3)(2 * 5 * 64, 5 * 64, 64)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _pool(**kw):
    p = ob.PagePool()
    p.K = p.V = p.page_table = FAKE
    p.n_pages, p.page_rows, p.pages_cap = 32, 16, 8
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _layer():
    d = ob.LayerDesc()
    d.batch, d.n_q_heads, d.n_kv_heads, d.head_dim, d.n_tokens = 1, 4, 2, 64, 30
    d.vis_begin, d.vis_end, d.causal, d.dtype, d.softmax_scale = 0, 20, 1, ob.OMNI_F32, 0.125
    d.q_stride = (C.c_int64 * 3)(4 * 30 * 64, 30 * 64, 64)
    d.kv_stride = (C.c_int64 * 3)(2 * 30 * 64, 30 * 64, 64)
    return d


def _attn(lib, desc=None, pool=None, Q=FAKE, row_end=FAKE, new_cnt=FAKE, O=2 * FAKE, lse=FAKE, acc_in=None, acc_out=None, ws=FAKE, n=BIG):
    desc, pool = desc or _chunk(), pool or _pool()
    return lib.omni_paged_attn(C.byref(desc), Q, C.byref(pool), row_end, new_cnt, O, lse, acc_in, acc_out, ws, n, None)


def _append(lib, desc=None, rope=None, pool=None, Q=None, K=FAKE, V=FAKE, pos=FAKE, new_cnt=FAKE, row_cnt=FAKE, Qout=None,
            row_end=2 * FAKE, row_pos=FAKE, acc=None):
    desc, pool = desc or _chunk(), pool or _pool()
    return lib.omni_paged_append(C.byref(desc), None if rope is None else C.byref(rope), Q, K, V, C.byref(pool), pos, new_cnt,
                                 row_cnt, Qout, row_end, row_pos, acc, None)


def _evict(lib, desc=None, pool=None, budget=8, sink=1, recent=2, seq_len=FAKE, ws=FAKE, n=BIG, row_cnt=FAKE):
    desc, pool = desc or _chunk(), pool or _pool()
    return lib.omni_paged_evict(C.byref(desc), C.byref(pool), budget, sink, recent, seq_len, FAKE, FAKE, FAKE, row_cnt, FAKE, FAKE,
                                ws, n, None)


@pytest.mark.parametrize("kw,code,needle", [
    (dict(head_dim=96), -2, "head_dim"), (dict(n_kv_heads=3), -1, "multiple"), (dict(dtype=5), -2, "dtype"),
    (dict(n_new=0), -1, "positive"), (dict(batch=0), -1, "positive"), (dict(causal=2), -1, "causal"),
    (dict(softmax_scale=float("nan")), -1, "softmax_scale"), (dict(softmax_scale=-1.0), -1, "softmax_scale"),
    (dict(q_stride=(C.c_int64 * 3)(1280, 320, 60)), -1, "multiples of 8"),
    (dict(q_stride=(C.c_int64 * 3)(0, 320, 64)), -1, "at least head_dim"),
    (dict(kv_stride=(C.c_int64 * 3)(640, 320, 32)), -1, "at least head_dim"),
    (dict(batch=20000), -2, "65535"), (dict(n_new=1 << 29), -2, "2^31"),
])
def test_chunk_descriptors_that_are_refused(lib, kw, code, needle):
    d = _chunk(**kw)
    for call in (_attn, _append, _evict):
        assert call(lib, desc=d) == code
        assert needle in ob.last_error()
    with pytest.raises(ob.OmniError):
        ob.workspace_bytes(ob.CALL_PAGED_ATTN, d, 128)


@pytest.mark.parametrize("kw,code,needle", [
    (dict(K=None), -1, "null"), (dict(V=FAKE + 8), -1, "aligned"), (dict(page_table=None), -1, "null"),
    (dict(page_rows=24), -2, "power of two"), (dict(n_pages=0), -1, ">= 1"), (dict(pages_cap=0), -1, ">= 1"),
    (dict(n_pages=1 << 27), -2, "2^31"), (dict(pages_cap=1 << 27), -2, "2^30"),
])
def test_pools_that_are_refused(lib, kw, code, needle):
    for call in (_attn, _append, _evict):
        assert call(lib, pool=_pool(**kw)) == code
        assert needle in ob.last_error()


def test_attention_refuses(lib):
    assert _attn(lib, pool=_pool(page_rows=8)) == -2 and "16" in ob.last_error()
    for kw in ("Q", "row_end", "new_cnt", "O", "lse", "ws"):
        assert _attn(lib, **{kw: None}) == -1 and "null" in ob.last_error()
    assert _attn(lib, Q=FAKE + 8) == -1 and _attn(lib, O=FAKE + 8) == -1
    assert _attn(lib, O=FAKE) == -1 and "O must not be Q" in ob.last_error()
    assert _attn(lib, acc_in=FAKE) == -1 and "acc_out" in ob.last_error()
    assert _attn(lib, acc_out=FAKE + 4) == -1 and "aligned" in ob.last_error()
    assert _attn(lib, ws=FAKE + 16) == -3 and _attn(lib, n=0) == -3
    need = ob.workspace_bytes(ob.CALL_PAGED_ATTN, _chunk(), 128)
    assert _attn(lib, acc_out=FAKE, n=need - 1) == -3
    with pytest.raises(ob.OmniError):
        ob.workspace_bytes(ob.CALL_PAGED_ATTN, _chunk(), -1)


def test_append_refuses(lib):
    rope = ob.make_rope_desc(64)
    for kw in ("K", "V", "pos", "new_cnt", "row_cnt", "row_end", "row_pos"):
        assert _append(lib, **{kw: None}) == -1 and "null" in ob.last_error()
    assert _append(lib, rope=rope, Q=FAKE) == -1 and _append(lib, rope=rope, Qout=FAKE) == -1
    assert _append(lib, Q=FAKE, Qout=FAKE) == -1 and "rope" in ob.last_error()
    assert _append(lib, row_end=FAKE) == -1 and "row_end" in ob.last_error()
    assert _append(lib, K=FAKE + 4) == -1
    assert _append(lib, rope=ob.make_rope_desc(128), Q=FAKE, Qout=FAKE) == -1 and "head_dim" in ob.last_error()
    assert _append(lib, rope=ob.RopeDesc(64, 24, 0, 1.0), Q=FAKE, Qout=FAKE) == -2 and "rot_dim" in ob.last_error()


def test_eviction_refuses(lib):
    assert _evict(lib, budget=0, sink=0, recent=0) == -1 and _evict(lib, budget=2) == -1 and "budget" in ob.last_error()
    assert _evict(lib, budget=2 ** 31 - 1, sink=2 ** 31 - 1, recent=2 ** 31 - 1) == -1
    assert _evict(lib, sink=-1) == -1 and _evict(lib, recent=-1) == -1
    assert _evict(lib, seq_len=None) == -1 and _evict(lib, row_cnt=None) == -1
    assert _evict(lib, n=0) == -3 and _evict(lib, ws=None) == -1
    assert ob.workspace_bytes(ob.CALL_PAGED_EVICT, _chunk(), 128) > 0


def test_rope_refuses(lib):
    d, r = _layer(), ob.make_rope_desc(64)
    call = lambda rope=r, desc=d, Q=FAKE, back=0, Qout=FAKE: lib.omni_rope(  # noqa: E731
        C.byref(rope), C.byref(desc), Q, FAKE, None, back, Qout, FAKE, None)
    assert call(Q=None) == -1 and call(Qout=None) == -1 and call(Q=FAKE + 4) == -1 and call(back=2) == -1
    assert call(rope=ob.make_rope_desc(128)) == -1
    bad = ob.make_rope_desc(64)
    bad.inv_freq[3] = float("nan")
    assert call(rope=bad) == -1 and "inv_freq" in ob.last_error()
    bad = ob.make_rope_desc(64)
    bad.interleaved = 2
    assert call(rope=bad) == -1


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=20), dict(rot_dim=80), dict(base=1.0), dict(base=float("inf")),
                                dict(scaling="linear", factor=0.0), dict(scaling="linear", factor=float("nan")),
                                dict(scaling="by_parts", factor=2.0), dict(scaling="by_parts", factor=2.0, orig_len=10, low_turns=3, high_turns=3)])
def test_rope_plans_that_are_refused(kw):
    with pytest.raises(ob.OmniError):
        ob.make_rope_desc(64, **kw)


def test_rope_plan_names():
    with pytest.raises(ValueError):
        ob.make_rope_desc(64, scaling="other")
    with pytest.raises(ob.OmniError):
        ob.make_rope_desc(96)


@pytest.mark.parametrize("kw", [dict(), dict(base=1e6), dict(scaling="linear", factor=8.0),
                                dict(scaling="by_parts", factor=4.0, orig_len=4096, low_turns=2, high_turns=20)])
@pytest.mark.parametrize("rot", [16, 64, 128])
def test_rope_frequencies(rot, kw):
    got = ob.make_rope_desc(128, rot, **kw)
    # a handful of roundings of 2^-53 each, pow among them
    np.testing.assert_allclose(got.inv_freq[:rot // 2], po.rope_frequencies(rot, **kw), rtol=1e-14)


def test_tensors_that_the_binding_refuses():
    dt = torch.bfloat16
    Q, K = torch.zeros(2, 4, 5, 64, dtype=dt), torch.zeros(2, 2, 5, 64, dtype=dt)
    pages, table = torch.zeros(8, 16, 64, dtype=dt), torch.zeros(2, 2, 2, dtype=torch.int32)
    pool, desc = ob.make_page_pool(pages, pages.clone(), table), ob.make_chunk_desc(Q, K)
    ints, cnt = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    rows = torch.zeros(2, 2, 32, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        ob.omni_paged_attn(desc, Q, pool, ints, cnt)
    with pytest.raises(ValueError, match="row_end"):
        ob.omni_paged_attn(desc, Q, pool, ints.long(), cnt)
    with pytest.raises(ValueError, match="new_cnt"):
        ob.omni_paged_attn(desc, Q, pool, ints, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="strides"):
        ob.omni_paged_attn(desc, Q.transpose(1, 2).contiguous().transpose(1, 2), pool, ints, cnt)
    with pytest.raises(ValueError, match="acc_out"):
        ob.omni_paged_attn(desc, Q, pool, ints, cnt, acc_out=torch.zeros(2, 2, 31))
    with pytest.raises(ValueError, match="pool dtype"):
        ob.omni_paged_attn(ob.make_chunk_desc(Q.float(), K.float()), Q.float(), pool, ints, cnt)
    with pytest.raises(ValueError, match="pairs"):
        ob.omni_paged_attn(ob.make_chunk_desc(Q[:1], K[:1]), Q[:1], pool, ints[:1], cnt[:1])
    with pytest.raises(ValueError, match="row_pos"):
        ob.omni_paged_append(desc, None, None, K, K, pool, cnt, cnt, ints, rows[..., :16])
    with pytest.raises(ValueError, match="rope"):
        ob.omni_paged_append(desc, None, Q, K, K, pool, cnt, cnt, ints, rows)
    with pytest.raises(ValueError, match="seq_len"):
        ob.omni_paged_evict(pool, 4, 0, 0, ints, ints, rows, rows.float())
    with pytest.raises(ValueError, match="head_dim"):
        ob.make_chunk_desc(Q.transpose(2, 3), K)
    with pytest.raises(ValueError, match="K must"):
        ob.make_chunk_desc(Q, K[:, :, :4])
    with pytest.raises(ValueError, match="give K"):
        ob.make_chunk_desc(Q)


def test_strides_of_single_element_dimensions_do_not_matter():
    q = torch.zeros(1, 4, 64).as_strided((1, 4, 1, 64), (7, 64, 3, 1))
    d = ob.make_chunk_desc(q, n_kv_heads=2)
    assert list(d.q_stride) == [256, 64, 64] and list(d.kv_stride) == [128, 64, 64]
