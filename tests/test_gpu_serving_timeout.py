"""Waits that run out in the calls without a context: reported, NaN in what is concerned, nothing hangs, and the next call is right.

The knob d2o_set_static_fault_injection shortens the limit to two milliseconds, keeps copies from being issued, and counts answers as late."""
import time

import pytest
import torch

from paper_2406_13035_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16}
D2O_ERR_TIMEOUT = 6


@pytest.fixture
def knob():
    yield B.d2o_set_static_fault_injection
    B.d2o_set_static_fault_injection()


def _prompt(dtype, d, b, hq, hkv, n):
    g = torch.Generator(device="cuda").manual_seed(n)
    return [torch.randn(b, h, n, d, generator=g, device="cuda").to(DT[dtype]) for h in (hq, hkv, hkv)]


def _timed(call):
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    call()
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 < 1.0


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("b,hq,hkv,n,lens", [(4, 64, 8, 600, [600, 300, 0, 257]), (1, 3, 3, 400, [400]), (3, 40, 8, 1500, [1500, 700, 1])])
def test_prompt_attention_answers_that_come_late(cuda_device, knob, dtype, d, b, hq, hkv, n, lens):
    """The work that a thread block took over without learning of it in time is NaN like its own: no row keeps what it held."""
    q, k, v = _prompt(dtype, d, b, hq, hkv, n)
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = torch.full_like(q, 7.0)
    B.d2o_prompt_attention(q, k, v, want, lens=dl)
    out, lse = torch.full_like(q, 7.0), torch.full((b, hq, n), 7.0, device="cuda")
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    knob(2000, -1, True)
    _timed(lambda: B.d2o_prompt_attention(q, k, v, out, lse=lse, lens=dl, status=status))
    assert status.tolist()[0] == D2O_ERR_TIMEOUT
    for i, m in enumerate(lens):
        assert bool(out[i, :, :m].isnan().all()) and bool(lse[i, :, :m].isnan().all()), i
        assert bool((out[i, :, m:] == 7).all()) and bool((lse[i, :, m:] == 7).all()), i
    knob()
    status.zero_()
    B.d2o_prompt_attention(q, k, v, out.fill_(7.0), lens=dl, status=status)
    assert torch.equal(out, want) and status.tolist() == [0, 0]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("stage", [0, 1, 4, 9, 17])
def test_prompt_attention_whose_tiles_do_not_arrive(cuda_device, knob, dtype, d, stage):
    """Every row is NaN or right, and those that needed the tiles are NaN."""
    b, hq, hkv, n = 2, 48, 8, 1300
    q, k, v = _prompt(dtype, d, b, hq, hkv, n)
    want, out = torch.empty_like(q), torch.full_like(q, 7.0)
    B.d2o_prompt_attention(q, k, v, want)
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    knob(2000, stage)
    _timed(lambda: B.d2o_prompt_attention(q, k, v, out, status=status))
    assert status.tolist()[0] == D2O_ERR_TIMEOUT
    bad = out.isnan()
    assert bool((bad | (out == want)).all()) and bool((bad.all(-1) == bad.any(-1)).all())
    assert bool(bad[:, :, 1280:].all())                        # the last block, which sees 22 tiles of keys and values
    knob()
    B.d2o_prompt_attention(q, k, v, out)
    assert torch.equal(out, want)
