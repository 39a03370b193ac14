"""Host checks of the serving entry points, without a GPU: every refusal comes back before anything is enqueued."""
import ctypes

import pytest
import torch

from paper_2510_13161_amd import msd

A = 0x1000  # an aligned address that no refused call reads


def cache(**kw):
    c = msd.PagedKV(A, A, A, A, A, A, A, msd.MSD_KV_FP8, 2, 8, 4, 64, 128, 3, 5)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows(**kw):
    r = msd.KVRows(A, A, 0, 1024, 512, 128, 0, 1, 2, 7, None)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def rope(**kw):
    r = msd.Rope(A, 320, 128, 0)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def attn(**kw):
    a = msd.PagedAttn(A, 4096, 1024, 128, A, 4096, 1024, 128, None, None, 0, 0, 0, None, None, None, 0.1, 2, 4, 8, 0, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def refused(rc, status):
    assert rc == status, (rc, msd.last_error())
    assert msd.last_error()


BAD_CACHE = [({"k": None}, -1), ({"v": None}, -1), ({"page_table": None}, -1), ({"len": None}, -1), ({"status": None}, -1),
             ({"k_scale": None}, -1), ({"v_scale": None}, -1), ({"k": A + 8}, -1), ({"format": 2}, -4),
             ({"head_dim": 96}, -2), ({"page_size": 48}, -2), ({"page_size": 8}, -2), ({"page_size": 512}, -2),
             ({"n_pages": 0}, -2), ({"n_layers": 0}, -2), ({"n_kv_heads": 0}, -2), ({"batch_cap": 0}, -2),
             ({"max_pages": 0}, -2), ({"max_pages": 1 << 25}, -3)]


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_every_call_refuses_a_bad_cache(kw, status):
    L, c = msd.lib(), cache(**kw)
    refused(L.msd_paged_append(ctypes.byref(c), ctypes.byref(rows()), None, None), status)
    refused(L.msd_paged_commit(ctypes.byref(c), ctypes.byref(rows(n_layers=2)), None, A, A, None), status)
    refused(L.msd_paged_attention(ctypes.byref(c), 0, ctypes.byref(attn()), A, 1 << 40, None), status)


BAD_ROWS = [({"k": None}, -1), ({"v": None}, -1), ({"k": A + 2}, -1), ({"row_stride": 129}, -2), ({"head_stride": -8}, -2),
            ({"seq_stride": 4}, -2), ({"layer_stride": 12}, -2), ({"layer": -1}, -2), ({"layer": 2}, -2), ({"n_layers": 0}, -2),
            ({"n_layers": 3}, -2), ({"batch": 0}, -2), ({"batch": 4}, -2), ({"n_rows": 0}, -3), ({"n_rows": 321}, -3)]


@pytest.mark.parametrize("kw,status", BAD_ROWS)
def test_append_refuses_bad_rows(kw, status):
    refused(msd.lib().msd_paged_append(ctypes.byref(cache()), ctypes.byref(rows(**kw)), None, None), status)


BAD_ROPE = [({"table": None}, -1), ({"table": A + 4}, -1), ({"layout": 2}, -1), ({"rotary_dim": 8}, -2),
            ({"rotary_dim": 24}, -2), ({"rotary_dim": 144}, -2), ({"positions": 319}, -3)]


@pytest.mark.parametrize("kw,status", BAD_ROPE)
def test_bad_rotations_are_refused(kw, status):
    L, r = msd.lib(), rope(**kw)
    refused(L.msd_paged_append(ctypes.byref(cache()), ctypes.byref(rows()), ctypes.byref(r), None), status)
    a = attn(rope=ctypes.pointer(r))
    refused(L.msd_paged_attention(ctypes.byref(cache()), 0, ctypes.byref(a), A, 1 << 40, None), status)


def test_commit_refusals():
    L, c = msd.lib(), cache()
    ok = dict(n_layers=2)
    for r, acc, path, status in [(rows(**ok), None, A, -1), (rows(**ok), A, None, -1), (rows(count=A, **ok), A, A, -1),
                                 (rows(n_rows=65, **ok), A, A, -2), (rows(), A, A, -2), (rows(layer=1), A, A, -2)]:
        refused(L.msd_paged_commit(ctypes.byref(c), ctypes.byref(r), None, acc, path, None), status)


BAD_ATTN = [({"q": None}, -1), ({"out": None}, -1), ({"k_new": A}, -1), ({"v_new": A}, -1), ({"q": A + 2}, -1),
            ({"k_new": A, "v_new": A + 8}, -1), ({"q_row": 4}, -2), ({"out_head": -8}, -2), ({"new_seq": 2}, -2),
            ({"batch": 0}, -2), ({"batch": 4}, -2), ({"n_slots": 0}, -2), ({"n_slots": 65}, -2), ({"n_heads": 6}, -2),
            ({"n_heads": 0}, -2), ({"scale": float("inf")}, -1), ({"scale": float("nan")}, -1), ({"window": -1}, -1),
            ({"sinks": -1}, -1)]


@pytest.mark.parametrize("kw,status", BAD_ATTN)
def test_attention_refuses_bad_arguments(kw, status):
    refused(msd.lib().msd_paged_attention(ctypes.byref(cache()), 0, ctypes.byref(attn(**kw)), A, 1 << 40, None), status)


def test_attention_refuses_layers_trees_and_workspaces():
    L, c = msd.lib(), cache()
    for layer in (-1, 2):
        refused(L.msd_paged_attention(ctypes.byref(c), layer, ctypes.byref(attn()), A, 1 << 40, None), -2)
    tree = (ctypes.c_int32 * 4)(-1, 0, 0, 1)
    p = ctypes.cast(tree, ctypes.POINTER(ctypes.c_int32))
    refused(L.msd_paged_attention(ctypes.byref(c), 0, ctypes.byref(attn(parent=p)), A, 1 << 40, None), -4)
    for bad in ((0, 0, 0, 1), (-1, 1, 0, 0), (-1, -1, 0, 0), (-1, 0, 3, 0)):
        t = (ctypes.c_int32 * 4)(*bad)
        a = attn(parent=ctypes.cast(t, ctypes.POINTER(ctypes.c_int32)), k_new=A, v_new=A)
        refused(L.msd_paged_attention(ctypes.byref(c), 0, ctypes.byref(a), A, 1 << 40, None), -2)
    need = L.msd_paged_attention_workspace_bytes(ctypes.byref(c), 2, 4, 8)
    for ws, nb in ((None, need), (A, need - 1), (A + 4, need)):
        refused(L.msd_paged_attention(ctypes.byref(c), 0, ctypes.byref(attn()), ws, nb, None), -5)
    small = cache(page_size=16, max_pages=1)
    refused(L.msd_paged_attention(ctypes.byref(small), 0, ctypes.byref(attn(n_slots=17)), A, 1 << 40, None), -3)


def test_null_structs_are_refused():
    L, c = msd.lib(), cache()
    refused(L.msd_paged_append(None, ctypes.byref(rows()), None, None), -1)
    refused(L.msd_paged_append(ctypes.byref(c), None, None, None), -1)
    refused(L.msd_paged_commit(ctypes.byref(c), None, None, A, A, None), -1)
    refused(L.msd_paged_attention(ctypes.byref(c), 0, None, A, 1 << 40, None), -1)
    assert L.msd_paged_attention_workspace_bytes(None, 1, 1, 1) == 0
    assert L.msd_paged_attention_workspace_bytes(ctypes.byref(c), 0, 1, 1) == 0
    assert L.msd_sample_workspace_bytes(0, 5) == 0 and L.msd_sample_workspace_bytes(5, 0) == 0


def test_attention_workspace_never_falls():
    L, c = msd.lib(), cache()
    for batch in (1, 2, 5, 16, 40):
        for n in (1, 2, 9, 25, 64):
            for heads in (4, 20, 40):
                x = L.msd_paged_attention_workspace_bytes(ctypes.byref(c), batch, n, heads)
                assert x > 0
                assert L.msd_paged_attention_workspace_bytes(ctypes.byref(c), batch + 1, n, heads) >= x
                assert L.msd_paged_attention_workspace_bytes(ctypes.byref(c), batch, min(n + 1, 64), heads) >= x
                assert L.msd_paged_attention_workspace_bytes(ctypes.byref(c), batch, n, heads + 4) >= x


def test_sample_workspace_never_falls():
    f = msd.lib().msd_sample_workspace_bytes
    for rows in (1, 5, 13, 14, 60, 144, 65535):
        for vocab in (1, 2047, 2049, 8192, 8193, 32000, 152064, 524288, 524289, 1048575):
            assert 0 < f(rows, vocab) <= f(rows + 1, vocab) and f(rows, vocab) <= f(rows, vocab + 1)


@pytest.mark.parametrize("kw,status", [({"logits": None}, -1), ({"u": None}, -1), ({"tok": None}, -1), ({"rows": 0}, -2),
                                       ({"rows": 65536}, -2), ({"vocab": 0}, -2), ({"vocab": 1048577}, -2),
                                       ({"stride": 99}, -2), ({"ws": None}, -5), ({"ws": A + 8}, -5), ({"nb": 0}, -5)])
def test_sample_refuses(kw, status):
    d = dict(logits=A, stride=1048577 if kw.get("vocab", 0) > 1048576 else 100, rows=3, vocab=100, u=A, tok=A, ws=A, nb=1 << 40)
    d.update(kw)
    refused(msd.lib().msd_sample(d["logits"], d["stride"], d["rows"], d["vocab"], None, d["u"], d["tok"], None, None, d["ws"],
                                 d["nb"], None), status)


def test_binding_refuses_tensors_that_do_not_fit():
    x = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(msd.MsdError):      # not on the device
        msd.kv_rows(x, x)
    with pytest.raises(msd.MsdError):
        msd.paged_attn(x, x)
    with pytest.raises(msd.MsdError):
        msd.rope(torch.zeros(4, 8, 2), "spiral")
    with pytest.raises(msd.MsdError):
        msd.sample_params(temperature=torch.ones(3))
    with pytest.raises(msd.MsdError):
        msd.PagedCache(x, x, x, x, x)


def test_struct_sizes():
    assert ctypes.sizeof(msd.PagedKV) == 7 * 8 + 8 * 4
    assert ctypes.sizeof(msd.Rope) == 8 + 3 * 4 + 4
    assert ctypes.sizeof(msd.KVRows) == 2 * 8 + 4 * 8 + 4 * 4 + 8
    assert ctypes.sizeof(msd.PagedAttn) == 13 * 8 + 3 * 8 + 4 + 5 * 4
    assert ctypes.sizeof(msd.SampleParams) == 4 * 8
