"""Host-side checks of the serving entry points (no GPU): bad arguments are rejected before anything is launched."""
import ctypes
import os

import pytest
import torch

from paper_2602_08426_amd import binding as pb

FAKE = 4096                       # an aligned address that is never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pb.library_path()):
        from paper_2602_08426_amd.build import build_library
        build_library()
    return pb._load()


def ref(x):
    return ctypes.byref(x) if x is not None else None


def rows(data=FAKE, head=128 * 10, token=128):
    return pb.prism_rows(data, head, token)


def rotary(**kw):
    base = dict(base=1e4, rot_dim=128)
    base.update(kw)
    return pb.make_rotary(**base)


def cache(**kw):
    base = dict(k=FAKE, v=FAKE, k_scale=None, v_scale=None, page_stride=0, n_pages=10, n_kv_heads=2, page=64, head_dim=128, dtype=0)
    base.update(kw)
    return pb.prism_cache(*(base[f] for f, _ in pb.prism_cache._fields_))


def batch(**kw):
    base = dict(n_seqs=2, n_tokens=10, max_tokens=5, max_pages=4, cu_tokens=None, lengths=FAKE, page_table=FAKE)
    base.update(kw)
    return pb.prism_batch(*(base[f] for f, _ in pb.prism_batch._fields_))


def params(**kw):
    base = dict(n_q_heads=8, window=0, sinks=0, scale=0.0)
    base.update(kw)
    return pb.prism_cache_attn_params(*(base[f] for f, _ in pb.prism_cache_attn_params._fields_))


BAD_ROTARY = [dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(rot_dim=0), dict(rot_dim=24), dict(rot_dim=144), dict(rot_dim=-16),
              dict(layout=2), dict(magnitude=0.0), dict(magnitude=float("nan")), dict(magnitude=float("inf")),
              dict(position_offset=-1), dict(position_offset=1 << 30), dict(yarn_native_len=-1),
              dict(yarn_native_len=4096, yarn_scale=0.5), dict(yarn_native_len=4096, yarn_alpha=4.0, yarn_beta=4.0),
              dict(yarn_native_len=4096, yarn_scale=float("inf"))]
BAD_ROWS = [dict(data=None), dict(data=FAKE + 8), dict(head=-8), dict(token=-128), dict(head=1284), dict(token=129), dict(head=1 << 61)]
BAD_OUT = [dict(head=0), dict(token=0), dict(token=64), dict(head=128, token=128), dict(head=1272, token=128), dict(head=128, token=136)]
BAD_CACHE = [(dict(page=16), -2), (dict(page=48), -2), (dict(page=256), -2), (dict(head_dim=96), -2), (dict(dtype=2), -2), (dict(n_pages=0), -1), (dict(n_kv_heads=0), -1),
             (dict(page_stride=2 * 64 * 128 - 16), -1), (dict(page_stride=2 * 64 * 128 + 8), -1), (dict(page_stride=-16), -1),
             (dict(page_stride=1 << 60), -1)]
BAD_MEMORY = [dict(k=None), dict(v=None), dict(k=FAKE + 2), dict(k_scale=FAKE), dict(dtype=1), dict(dtype=1, k_scale=FAKE)]
BAD_BATCH = [(dict(n_seqs=-1), -1), (dict(n_tokens=-1), -1), (dict(max_tokens=0), -1), (dict(max_pages=0), -1), (dict(n_seqs=0), -1), (dict(lengths=None), -1),
             (dict(page_table=None), -1), (dict(n_tokens=9), -1), (dict(max_pages=(1 << 23) + 1), -2), (dict(n_tokens=(1 << 27) + 1, cu_tokens=FAKE), -2),
             (dict(n_seqs=(1 << 21) + 1, cu_tokens=FAKE), -2)]


def rotate(lib, r=None, d=128, n=10, h=4, q=None, qo=None, h_kv=2, k=None, ko=None, flags=0):
    r = rotary() if r is None else r
    q, qo, k, ko = (rows() if x is None else x for x in (q, qo, k, ko))
    return lib.prism_rotate(ref(r), d, n, None, h, ref(q), ref(qo), h_kv, ref(k), ref(ko), flags, None)


def test_rotate_refusals(lib):
    for kw in BAD_ROTARY:
        assert rotate(lib, rotary(**kw)) == -1, kw
    assert lib.prism_rotate(None, 128, 10, None, 4, ref(rows()), ref(rows()), 0, None, None, 0, None) == -1
    for kw in BAD_ROWS:
        for side in ("q", "qo", "k", "ko"):
            assert rotate(lib, **{side: rows(**kw)}) == -1, (side, kw)
    for kw in BAD_OUT:
        for side in ("qo", "ko"):
            assert rotate(lib, **{side: rows(data=FAKE * 2, **kw)}, n=10, h=4) == -1, (side, kw)
    assert rotate(lib, d=96) == -2 and rotate(lib, n=-1) == -1 and rotate(lib, h=-1) == -1 and rotate(lib, flags=2) == -1
    assert rotate(lib, n=(1 << 27) + 1) == -2 and rotate(lib, h=(1 << 16) + 1) == -2
    assert rotate(lib, q=rows(token=256, head=2560)) == -1                    # starts as its output, other strides
    assert lib.prism_rotate(ref(rotary()), 128, 10, None, 4, None, ref(rows()), 0, None, None, 0, None) == -1


def append(lib, c=None, b=None, r=None, k=None, v=None, h=0, q=None, qo=None):
    c, b = cache() if c is None else c, batch() if b is None else b
    k, v = (rows() if x is None else x for x in (k, v))
    return lib.prism_cache_append(ref(c), ref(b), ref(r), ref(k), ref(v), h, ref(q), ref(qo), None)


def attn(lib, c=None, b=None, p=None, q=None, out=None, ws=FAKE, size=1 << 40):
    c, b, p = cache() if c is None else c, batch() if b is None else b, params() if p is None else p
    q, out = (rows() if x is None else x for x in (q, out))
    return lib.prism_cache_attn(ref(c), ref(b), ref(p), ref(q), ref(out), None, ws, size, None)


def test_cache_and_batch_refusals(lib):
    n = ctypes.c_size_t(0)
    size = lambda c, b: lib.prism_cache_attn_workspace_bytes(ref(c), ref(b), 8, ctypes.byref(n))
    for call in (lambda c, b: append(lib, c, b), lambda c, b: attn(lib, c, b), size):
        for kw, rc in BAD_CACHE:
            assert call(cache(**kw), batch()) == rc, kw
        for kw, rc in BAD_BATCH:
            assert call(cache(), batch(**kw)) == rc, kw
    for kw in BAD_MEMORY:
        assert append(lib, cache(**kw)) == -1 and attn(lib, cache(**kw)) == -1, kw
    assert lib.prism_cache_append(None, ref(batch()), None, ref(rows()), ref(rows()), 0, None, None, None) == -1
    assert lib.prism_cache_append(ref(cache()), None, None, ref(rows()), ref(rows()), 0, None, None, None) == -1
    assert lib.prism_cache_attn(ref(cache()), ref(batch()), None, ref(rows()), ref(rows()), None, FAKE, 1 << 40, None) == -1


def test_append_refusals(lib):
    for kw in BAD_ROTARY:
        assert append(lib, r=rotary(**kw)) == -1, kw
    for kw in BAD_ROWS:
        for side in ("k", "v"):
            assert append(lib, **{side: rows(**kw)}) == -1, (side, kw)
        assert append(lib, r=rotary(), h=4, q=rows(**kw), qo=rows()) == -1, kw
        assert append(lib, r=rotary(), h=4, q=rows(data=FAKE * 2), qo=rows(**kw)) == -1, kw
    for kw in BAD_OUT:
        assert append(lib, r=rotary(), h=4, q=rows(), qo=rows(data=FAKE * 2, **kw)) == -1, kw
    assert append(lib, r=rotary(), h=4, q=rows()) == -1                       # Q without its output
    assert append(lib, h=4, qo=rows()) == -1
    assert append(lib, r=rotary(), h=0, q=rows(), qo=rows()) == -1
    assert append(lib, h=-1) == -1 and append(lib, h=(1 << 16) + 1) == -2
    assert append(lib, c=cache(n_kv_heads=(1 << 15) + 1)) == -2


def test_attention_refusals(lib):
    for kw in BAD_ROWS:
        assert attn(lib, q=rows(**kw)) == -1, kw
        assert attn(lib, out=rows(**kw)) == -1, kw
    for kw in BAD_OUT:
        assert attn(lib, out=rows(data=FAKE * 2, **kw)) == -1, kw
    for kw in (dict(n_q_heads=0), dict(n_q_heads=7), dict(window=-1), dict(sinks=-1), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert attn(lib, p=params(**kw)) == -1, kw
    assert attn(lib, ws=None) == -3 and attn(lib, ws=FAKE + 64) == -3 and attn(lib, size=16) == -3
    assert attn(lib, q=rows(token=256, head=2560)) == -1                      # starts as its output, other strides
    assert lib.prism_cache_attn_workspace_bytes(ref(cache()), ref(batch()), 8, None) == -1
    n = ctypes.c_size_t(0)
    size = lambda h, **kw: lib.prism_cache_attn_workspace_bytes(ref(cache()), ref(batch(cu_tokens=FAKE, **kw)), h, ctypes.byref(n))
    assert size(8, n_tokens=1 << 27) == 0 and size(10, n_tokens=1 << 27) == -2        # rows
    assert size(8, n_seqs=1 << 21) == 0
    assert lib.prism_cache_attn_workspace_bytes(ref(cache(n_kv_heads=4)), ref(batch(n_seqs=1 << 21, cu_tokens=FAKE)), 8, ctypes.byref(n)) == -2


def test_nothing_to_do_is_no_error(lib):
    none = batch(n_seqs=0, n_tokens=0, lengths=None, page_table=None)
    assert append(lib, b=none) == 0 and attn(lib, b=none, ws=None, size=0) == 0
    assert rotate(lib, n=0) == 0 and rotate(lib, h=0, h_kv=0) == 0


def test_binding_refuses_descriptors_of_another_device(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    x = torch.zeros((2, 10, 128), dtype=torch.bfloat16)
    for there in ((1, 0), (0, 1)):
        c, b = cache(), batch()
        c._device, b._device = there
        for call in (lambda: pb.prism_cache_append(c, b, None, x, x), lambda: pb.prism_cache_attn(c, b, x, x, None, x)):
            with pytest.raises(ValueError, match="current device"):
                call()


def test_binding_refuses_what_is_not_on_the_device():
    x = torch.zeros((2, 3, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        pb.prism_rotate(rotary(rot_dim=64), x, None, x, None)
    with pytest.raises(ValueError):
        pb.prism_rotate(rotary(rot_dim=64), None, None, None, None)
    with pytest.raises(ValueError):
        pb.prism_rotate(rotary(rot_dim=64), x, None, None, None)
    pages = torch.zeros((2, 1, 32, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        pb.make_cache(pages, pages)
    with pytest.raises(ValueError):
        pb.make_cache(pages.float(), pages.float())
    with pytest.raises(ValueError):
        pb.make_batch(torch.zeros(2, dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32))
    with pytest.raises(ValueError):
        pb.make_batch(torch.zeros(2, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32))
