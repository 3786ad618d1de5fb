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
    knob(2000, -1, 1)
    _timed(lambda: B.d2o_prompt_attention(q, k, v, out, lse=lse, lens=dl, status=status))
    assert status.tolist()[0] == D2O_ERR_TIMEOUT
    for i, m in enumerate(lens):
        assert bool(out[i, :, :m].isnan().all()) and bool(lse[i, :, :m].isnan().all()), i
        assert bool((out[i, :, m:] == 7).all()) and bool((lse[i, :, m:] == 7).all()), i
    knob()
    status.zero_()
    B.d2o_prompt_attention(q, k, v, out.fill_(7.0), lens=dl, status=status)
    assert torch.equal(out, want) and status.tolist() == [0, 0]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("f16", 128), ("bf16", 64)])
@pytest.mark.parametrize("b,hq,hkv,n", [(40, 64, 8, 100), (10, 64, 8, 300), (2, 40, 8, 1500)])
def test_prompt_attention_answers_that_come_late_later_on(cuda_device, knob, dtype, d, b, hq, hkv, n):
    """Blocks that go on for a while, and lose an answer while up to two items ahead of the one that it was asked behind are in work: every row is right or
    NaN, none keeps what it held."""
    q, k, v = _prompt(dtype, d, b, hq, hkv, n)
    want = torch.empty_like(q)
    B.d2o_prompt_attention(q, k, v, want)
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    for late in (2, 3, 4, 5) * 6:
        out, lse = torch.full_like(q, 7.0), torch.full((b, hq, n), 7.0, device="cuda")
        knob(2000, -1, late)
        _timed(lambda: B.d2o_prompt_attention(q, k, v, out, lse=lse, status=status))
        bad = out.isnan().all(-1)
        assert bool((bad | (out == want).all(-1)).all()) and torch.equal(bad, lse.isnan()), int((~bad & (out == 7.0).all(-1)).sum())


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


@pytest.mark.parametrize("dtype,d,G", [("bf16", 128, 4), ("f16", 64, 1), ("bf16", 64, 8), ("f16", 128, 2)])
@pytest.mark.parametrize("b,hkv,held,room", [(1, 4, 900, 1000), (2, 8, 300, 2000), (3, 8, 2500, 20000), (60, 8, 200, 400), (400, 2, 70, 100), (1, 1, 9000, 60000)])
@pytest.mark.parametrize("stage", [0, 1, 5, 13, 40])
def test_decode_step_whose_tiles_do_not_arrive(cuda_device, knob, dtype, d, G, b, hkv, held, room, stage):
    """One tile of every share is missing, in clusters and in shares of one or several slices: a slice's outputs are all NaN or right, never something
    else, and its scores are NaN where its outputs are.  The step after it is right, and the counters in the scratch are zero again."""
    page = 16
    g = torch.Generator(device="cuda").manual_seed(held + d)
    per, used = room // page, held // page + 1
    n_pages = b * used + 1
    table = torch.full((b, per), -1, dtype=torch.int32, device="cuda")
    table[:, :used] = torch.randperm(n_pages, generator=g, device="cuda")[: b * used].view(b, used).to(torch.int32)
    kp, vp = (torch.randn(n_pages, hkv, page, d, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    length = torch.randint(0, held + 1, (b, hkv), generator=g, device="cuda", dtype=torch.int32)
    length[0] = held
    q, k, v = (torch.randn(b, h, d, generator=g, device="cuda").to(DT[dtype]) for h in (hkv * G, hkv, hkv))
    pos, score = torch.zeros(n_pages, hkv, page, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, hkv, page, device="cuda")
    c = B.D2OPagedCache(kp, vp, table, length, n_q_heads=hkv * G, pos=pos, score=score)
    want, out = torch.empty_like(q), torch.full_like(q, 7.0)
    c.d2o_paged_decode_step(q, k, v, want)
    want_score = score.clone()
    c.check()
    score.zero_()
    knob(2000, stage)
    _timed(lambda: c.d2o_paged_decode_step(q, k, v, out))
    slices = lambda t: t.view(b, hkv, G * d)
    bad = slices(out).isnan()
    assert bool((bad.all(-1) == bad.any(-1)).all())
    bad = bad.all(-1)
    assert bool((bad | (slices(out) == slices(want)).all(-1)).all())
    dense = lambda t: t[table[:, :used].long()].transpose(1, 2).flatten(2)
    seen = torch.arange(used * page, device="cuda") <= length[..., None]
    got, was = dense(score), dense(want_score)
    assert bool((got.isnan() | ~seen)[bad].all()) and bool((got == was)[~bad].all()) and bool((got == 0)[~seen].all())
    if stage == 0:
        assert bool(bad.any())
    if bool(bad.any()):
        with pytest.raises(B.D2OError) as e:
            c.check()
        assert e.value.status == D2O_ERR_TIMEOUT
    else:
        c.check()
    knob()
    score.zero_()
    c.d2o_paged_decode_step(q, k, v, out)
    assert torch.equal(out, want) and torch.equal(score, want_score)
    c.check()
    zero = c._scratch[0] - c.scratch.data_ptr()
    assert not c.scratch[zero:zero + B.PAGED_ZERO_BYTES].any()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("f16", 128), ("bf16", 64)])
@pytest.mark.parametrize("b,hq,hkv,n", [(40, 64, 8, 100), (10, 64, 8, 300), (2, 40, 8, 1500), (1, 8, 8, 3000)])
def test_prompt_attention_with_hardly_any_patience(cuda_device, knob, dtype, d, b, hq, hkv, n):
    """Limits of a few microseconds, so that any wait runs out in any state of a block: every row is right or NaN, none keeps what it held; and the error
    word says so."""
    q, k, v = _prompt(dtype, d, b, hq, hkv, n)
    want = torch.empty_like(q)
    B.d2o_prompt_attention(q, k, v, want)
    failed = 0
    for limit in (1, 1, 1, 2, 2, 3, 3, 4, 5, 6, 8, 11, 15, 20):
        out, lse = torch.full_like(q, 7.0), torch.full((b, hq, n), 7.0, device="cuda")
        status = torch.zeros(2, dtype=torch.int32, device="cuda")
        knob(limit)
        _timed(lambda: B.d2o_prompt_attention(q, k, v, out, lse=lse, status=status))
        bad = out.isnan().all(-1)
        assert bool((bad | (out == want).all(-1)).all()) and torch.equal(bad, lse.isnan()), (limit, int((~bad & (out != want).any(-1)).sum()))
        assert status.tolist()[0] == D2O_ERR_TIMEOUT or not bool(bad.any())
        failed += bool(bad.any())
    assert failed
    knob()
    out = torch.empty_like(q)
    B.d2o_prompt_attention(q, k, v, out)
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype,d,G", [("bf16", 128, 4), ("f16", 64, 1), ("bf16", 64, 8), ("f16", 128, 2)])
@pytest.mark.parametrize("b,held,room", [(1, 900, 1000), (3, 2500, 20000), (60, 200, 400), (16, 3000, 6000)])
def test_decode_step_with_hardly_any_patience(cuda_device, knob, dtype, d, G, b, held, room):
    """The same for the decode step: every slice's outputs are right or NaN."""
    page, hkv = 16, 8
    g = torch.Generator(device="cuda").manual_seed(held + d)
    used = held // page + 1
    table = torch.full((b, room // page), -1, dtype=torch.int32, device="cuda")
    table[:, :used] = torch.randperm(b * used, generator=g, device="cuda").view(b, used).to(torch.int32)
    kp, vp = (torch.randn(b * used, hkv, page, d, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    length = torch.randint(0, held + 1, (b, hkv), generator=g, device="cuda", dtype=torch.int32)
    q, k, v = (torch.randn(b, h, d, generator=g, device="cuda").to(DT[dtype]) for h in (hkv * G, hkv, hkv))
    c = B.D2OPagedCache(kp, vp, table, length, n_q_heads=hkv * G)
    want = torch.empty_like(q)
    c.d2o_paged_decode_step(q, k, v, want)
    c.check()
    for limit in (1, 1, 1, 2, 2, 3, 4, 5, 6, 8, 11):
        flush = torch.zeros(1 << 28, dtype=torch.uint8, device="cuda")          # the rows come from memory
        out = torch.full_like(q, 7.0)
        knob(limit)
        _timed(lambda: c.d2o_paged_decode_step(q, k, v, out))
        bad = out.view(b * hkv, G * d).isnan()
        assert bool((bad.all(-1) == bad.any(-1)).all())
        right = (out.view(b * hkv, G * d) == want.view(b * hkv, G * d)).all(-1)
        assert bool((bad.all(-1) | right).all()), limit
        if bool(bad.any()):
            with pytest.raises(B.D2OError) as e:
                c.check()
            assert e.value.status == D2O_ERR_TIMEOUT
        c.status.zero_()
        del flush
    knob()
    out = torch.empty_like(q)
    c.d2o_paged_decode_step(q, k, v, out)
    assert torch.equal(out, want)
    c.check()
    zero = c._scratch[0] - c.scratch.data_ptr()
    assert not c.scratch[zero:zero + B.PAGED_ZERO_BYTES].any()
