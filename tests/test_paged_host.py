"""Arguments of the prompt attention and of the cache in pages that are refused before anything is launched (no GPU)."""
import ctypes as C

import pytest
import torch

from paper_2406_13035_b200 import binding as B
from paper_2406_13035_b200 import build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return B.load_library()


def cache(**kw):
    base = dict(dtype=2, d_head=128, batch=2, n_q_heads=8, n_kv_heads=2, page_size=16, n_pages=9, max_pages=4, k_pages=256,
                v_pages=256, pos=256, score=256, page_table=256, len=256, status=None)
    base.update(kw)
    return B.D2OPaged(*[base[f] for f, _ in B.D2OPaged._fields_])


BAD = [(dict(dtype=3), 2), (dict(d_head=96), 2), (dict(batch=0), 1), (dict(n_q_heads=7), 1), (dict(n_q_heads=6), 2), (dict(n_kv_heads=0), 1),
       (dict(page_size=8), 2), (dict(page_size=48), 2), (dict(page_size=2048), 2), (dict(n_pages=0), 1), (dict(max_pages=0), 1),
       (dict(n_pages=1 << 26), 2), (dict(max_pages=1 << 26), 2), (dict(batch=1 << 15), 2), (dict(pos=None), 1), (dict(score=None), 1)]


def test_workspace_size(lib):
    n = C.c_size_t()
    assert lib.d2o_paged_workspace_size(C.byref(cache()), C.byref(n)) == 0
    # with scores: four logits of 4 bytes, or a move of 8, per row of the pools
    m = C.c_size_t()
    assert lib.d2o_paged_workspace_size(C.byref(cache(pos=None, score=None)), C.byref(m)) == 0
    assert n.value - m.value == -(-9 * 2 * 16 * 16 // 256) * 256
    assert lib.d2o_paged_workspace_size(C.byref(cache(n_q_heads=2)), C.byref(n)) == 0
    assert lib.d2o_paged_workspace_size(None, C.byref(n)) == 1
    assert lib.d2o_paged_workspace_size(C.byref(cache()), None) == 1
    for kw, status in BAD:
        assert lib.d2o_paged_workspace_size(C.byref(cache(**kw)), C.byref(n)) == status, kw


def test_calls_refuse(lib):
    n = C.c_size_t()
    lib.d2o_paged_workspace_size(C.byref(cache()), C.byref(n))
    n = n.value
    append = lambda c, *a: lib.d2o_paged_append(C.byref(c), *a, None)
    step = lambda c, *a: lib.d2o_paged_decode_step(C.byref(c), *a, None)
    evict = lambda c, *a: lib.d2o_paged_evict(C.byref(c), *a, None)
    for kw, status in BAD + [(dict(k_pages=None), 1), (dict(v_pages=264), 1), (dict(page_table=None), 1), (dict(len=258), 1), (dict(len=None), 1),
                             (dict(status=257), 1), (dict(pos=257), 1)]:
        assert append(cache(**kw), 1, 256, 256, None, None, None) == status, kw
        assert step(cache(**kw), 0, 0, 256, 256, 256, None, 256, 256, n) == status, kw
        assert evict(cache(**kw), 256, 256, 0, 0, 256, n) == status, kw
    for n_rows in ((1 << 30) + 1, (1 << 31) - 1):
        assert append(cache(), n_rows, 256, 256, None, None, None) == 2
    bare = cache(pos=None, score=None)
    for a in [(0, 256, 256, None, None, None), (1, None, 256, None, None, None), (1, 256, 264, None, None, None), (1, 256, 256, 2, None, None)]:
        assert append(cache(), *a) == 1, a
    assert append(bare, 1, 256, 256, None, 256, None) == 1 and append(bare, 1, 256, 256, None, None, 256) == 1
    for a in [(-1, 0, 256, 256, 256, None, 256, 256, n), (0, -1, 256, 256, 256, None, 256, 256, n), (0, 0, None, 256, 256, None, 256, 256, n),
              (0, 0, 256, 8, 256, None, 256, 256, n), (0, 0, 256, 256, 256, 2, 256, 256, n), (0, 0, 256, 256, 256, None, None, 256, n),
              (0, 0, 256, 256, 256, None, 256, None, n)]:
        assert step(cache(), *a) == 1, a
    assert step(bare, 0, 0, 256, 256, 256, 256, 256, 256, n) == 1             # positions without pos
    assert step(cache(), 0, 0, 256, 256, 256, None, 256, 128, n) == 3         # misaligned scratch
    assert step(cache(), 0, 0, 256, 256, 256, None, 256, 256, n - 1) == 3
    for a in [(None, 256, 0, 0, 256, n), (256, None, 0, 0, 256, n), (256, 258, 0, 0, 256, n), (256, 256, -1, 0, 256, n), (256, 256, 0, -1, 256, n),
              (256, 256, 0, 0, None, n)]:
        assert evict(cache(), *a) == 1, a
    assert evict(bare, 256, 256, 0, 0, 256, n) == 1 and evict(cache(), 256, 256, 0, 0, 256, 16) == 3


def test_prompt_attention_refuses(lib):
    good = dict(dtype=2, d=128, b=1, hq=4, hkv=2, n=64, window=0, sinks=0, q=256, k=256, v=256, lens=None, out=256, lse=None, status=None)
    call = lambda **kw: lib.d2o_prompt_attention(*{**good, **kw}.values(), None)
    for kw, status in [(dict(dtype=5), 2), (dict(d=32), 2), (dict(b=0), 1), (dict(hq=0), 1), (dict(hkv=3), 1), (dict(n=0), 1), (dict(window=-1), 1),
                       (dict(sinks=-1), 1), (dict(q=None), 1), (dict(k=8), 1), (dict(v=None), 1), (dict(out=None), 1), (dict(lens=2), 1),
                       (dict(lse=1), 1), (dict(status=3), 1), (dict(n=(1 << 20) + 1), 2), (dict(b=1 << 12, n=1 << 20), 2)]:
        assert call(**kw) == status, kw


def test_binding_refuses_other_tensors():
    """Shapes, types, devices and strides are looked at before the library is called."""
    t = torch.zeros(1, 2, 8, 64)
    with pytest.raises(B.D2OError):
        B.d2o_prompt_attention(t, t, t, t)                                    # not on a GPU
    with pytest.raises(B.D2OError):
        B.D2OPagedCache(t, t, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32), n_q_heads=2)
    cpu = t.get_device()
    assert B._arg(None, "x", (1,), torch.float32, cpu) is None and B._arg(t, "x", t.shape, torch.float32, cpu) == t.data_ptr()
    for bad, shape, dtype, dev in [(t, (1, 2, 8, 32), torch.float32, cpu), (t, t.shape, torch.float16, cpu), (t, t.shape, torch.float32, 0),
                                   (t.transpose(1, 2), (1, 8, 2, 64), torch.float32, cpu)]:
        with pytest.raises(B.D2OError):
            B._arg(bad, "x", shape, dtype, dev)
    for view in [(-1, 0), (0, -1), (1 << 31, 0), (0, 1 << 32)]:
        with pytest.raises(B.D2OError):
            B._view(*view)
    assert B._view(0, (1 << 31) - 1) == (0, (1 << 31) - 1)
