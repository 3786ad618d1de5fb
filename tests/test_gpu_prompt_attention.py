"""d2o_prompt_attention against float64: lengths around its tiles, windows and sinks, ragged batches with anything in the padding,
grouped heads, both uses of its normalisers.

Tolerance.  A logit is a sum of d products in fp32; its error is a few 2^-24 of the magnitudes that it sums, at most
delta = 16 * 2^-24 * max_ij sum_e |q_ie k_je| / sqrt(d) (sixteen: partial sums of up to 16 elements at a time, four levels, and the
scale).  A weight is then off by a factor of at most 1 + 2 delta (itself and the sum), plus the rounding of exp2 and of the sum
(2^-21).  16-bit inputs: each weight is rounded once more for its product, by half a step.  So an output before its own rounding is
within e = (half a step of the weights' type + 2 delta + 2^-21) * sum_j p_ij |v_j| of the reference, and the result must be the
rounding of something in that interval.  lse is off by delta, and by the rounding of itself and of a logarithm (2^-22 of
max(1, |lse|))."""
import math

import pytest
import torch

from paper_2406_13035_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def reference(q, k, v, window, n_sink):
    """One head in float64: (out, lse, sum p |v|, sum |q||k| / sqrt d at most)."""
    q, k, v = q.double(), k.double(), v.double()
    n, d = q.shape
    i, j = torch.arange(n, device=q.device)[:, None], torch.arange(n, device=q.device)[None]
    seen = (j <= i) & ((j > i - window) | (j < n_sink)) if window > 0 else j <= i
    x = (q @ k.T / math.sqrt(d)).masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - lse[:, None])
    return p @ v, lse, p @ v.abs(), float((q.abs() @ k.abs().T).max()) / math.sqrt(d)


def check(q, k, v, out, lse, window, n_sink, dtype):
    ref, ref_lse, mag, dots = reference(q, k, v, window, n_sink)
    delta = 16 * 2.0 ** -24 * dots
    weights = 0.0 if dtype == "f32" else torch.finfo(DT[dtype]).eps / 2
    e = (weights + 2 * delta + 2.0 ** -21) * mag
    lo, hi, got = (ref - e).to(DT[dtype]).double(), (ref + e).to(DT[dtype]).double(), out.double()
    assert bool(((lo <= got) & (got <= hi)).all()), float(((got - ref).abs() / (e + ref.abs() * torch.finfo(DT[dtype]).eps)).max())
    if lse is not None:
        assert bool(((lse.double() - ref_lse).abs() <= delta + 2.0 ** -22 * ref_lse.abs().clamp(min=1)).all())


def draw(seed, b, hq, hkv, n, d, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda h: torch.randn(b, h, n, d, generator=g, device="cuda")
    return (r(hq) * scale).to(DT[dtype]), r(hkv).to(DT[dtype]), r(hkv).to(DT[dtype])


CASES = [  # batch, q heads, kv heads, d, tokens, window, sinks
    (1, 1, 1, 64, 1, 0, 0), (1, 2, 1, 128, 2, 1, 0), (2, 2, 2, 64, 63, 0, 0), (1, 4, 1, 128, 64, 16, 4), (1, 8, 1, 64, 65, 1, 1),
    (1, 3, 1, 128, 127, 64, 0), (1, 4, 4, 128, 128, 0, 0), (2, 4, 2, 64, 129, 128, 2), (1, 2, 2, 128, 255, 129, 130),
    (1, 2, 1, 128, 256, 0, 0), (1, 2, 1, 128, 257, 100, 0), (1, 2, 2, 64, 300, 1000, 4), (1, 8, 2, 128, 513, 77, 5),
    (1, 2, 2, 128, 700, 130, 300), (2, 4, 1, 64, 1000, 256, 1), (1, 4, 1, 128, 1153, 0, 0), (1, 2, 1, 128, 1500, 513, 129),
    (40, 8, 8, 64, 70, 0, 0), (2000, 4, 2, 64, 3, 0, 0), (1, 2, 1, 128, 640, 1, 0), (1, 1, 1, 64, 2050, 300, 7)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("b,hq,hkv,d,n,window,sinks", CASES)
def test_attention(cuda_device, b, hq, hkv, d, n, window, sinks, dtype):
    q, k, v = draw(n + window, b, hq, hkv, n, d, dtype)
    out, lse = torch.full_like(q, float("nan")), torch.full((b, hq, n), float("nan"), device="cuda")
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    B.d2o_prompt_attention(q, k, v, out, lse=lse, window=window, n_sink=sinks, status=status)
    for i in range(0, b, 13 if b < 100 else 333):
        for h in range(hq):
            check(q[i, h], k[i, h * hkv // hq], v[i, h * hkv // hq], out[i, h], lse[i, h], window, sinks, dtype)
    assert status.tolist() == [0, 0]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens,window,sinks", [([0, 1, 200, 128], 0, 0), ([257, 300, 5, 131], 70, 3), ([129, 64, 300, 0], 0, 0), ([-4, 999, 1, 250], 33, 0)])
def test_ragged(cuda_device, lens, window, sinks, dtype):
    """Padding holds NaN and infinities, in all three inputs; the rows of the outputs there stay as they were.  No lse."""
    n, d = 300, 128
    q, k, v = draw(n, 4, 4, 2, n, d, dtype)
    ends = [min(max(x, 0), n) for x in lens]
    for i, m in enumerate(ends):
        for t in (q, k, v):
            t[i, :, m:] = float("inf" if i % 2 else "nan")
    out = torch.full_like(q, 7.0)
    B.d2o_prompt_attention(q, k, v, out, window=window, n_sink=sinks, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    for i, m in enumerate(ends):
        assert bool((out[i, :, m:] == 7).all())
        for h in range(4 if m else 0):
            check(q[i, h, :m], k[i, h // 2, :m], v[i, h // 2, :m], out[i, h, :m], None, window, sinks, dtype)


@pytest.mark.parametrize("dtype,d", [("f16", 128), ("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("b,hq,hkv,n,window,sinks", [(2, 96, 8, 1100, 0, 0), (2, 96, 8, 1100, 300, 4), (5, 40, 40, 800, 0, 0), (5, 40, 40, 800, 150, 200)])
def test_more_blocks_than_places(cuda_device, dtype, d, b, hq, hkv, n, window, sinks):
    """Several blocks of queries for every SM, each of several tiles of keys and of lengths of their own, so that thread blocks go on with the work of others
    in every state of their rings."""
    q, k, v = draw(n + b, b, hq, hkv, n, d, dtype)
    lens = torch.tensor([n, n // 2 + 30, 1, n - 129, 257][:b], dtype=torch.int32)
    out, lse = torch.full_like(q, 7.0), torch.full((b, hq, n), 7.0, device="cuda")
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    B.d2o_prompt_attention(q, k, v, out, lse=lse, window=window, n_sink=sinks, lens=lens.cuda(), status=status)
    for i, m in enumerate(lens.tolist()):
        assert bool((out[i, :, m:] == 7).all()) and bool((lse[i, :, m:] == 7).all())
        for h in range(hq):
            check(q[i, h, :m], k[i, h * hkv // hq, :m], v[i, h * hkv // hq, :m], out[i, h, :m], lse[i, h, :m], window, sinks, dtype)
    assert status.tolist() == [0, 0]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_large_logits(cuda_device, dtype):
    """Logits in the hundreds that grow along the row, so that the running maximum moves in every tile, and fall, so that it never
    does: the weights of all but a few keys underflow."""
    n, d = 400, 64
    for sign in (1, -1):
        q, k, v = draw(5, 1, 1, 1, n, d, dtype)
        k = (k * 0.05 + sign * torch.arange(n, device="cuda")[:, None] * 0.02).to(DT[dtype])
        q = (q * 0.05 + 1.0).to(DT[dtype])
        out, lse = torch.empty_like(q), torch.empty(1, 1, n, device="cuda")
        B.d2o_prompt_attention(q, k, v, out, lse=lse)
        check(q[0, 0], k[0, 0], v[0, 0], out[0, 0], lse[0, 0], 0, 0, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("below", [18, 22, 24.4, 27.3, 30])
def test_many_small_weights_beside_a_large_one(cuda_device, dtype, d, below):
    """One key with nearly all of the weight and a value of nearly zero, and 20000 keys at 2^-below of it with values of one sign: what the small
    weights lose in their rounding does not average out.  Beyond the tolerance of the other tests an fp16 weight below 2^-21 of the row's largest is off by
    2^-32 of it (the largest is 2^7 at least, subnormals begin at 2^-14, and their half step is 2^-25)."""
    n = 20000
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k = (torch.zeros(1, 1, n, d, device="cuda") for _ in range(2))
    v = 4 + torch.rand(1, 1, n, d, generator=g, device="cuda")
    q[..., 0] = 4.0
    k[:, :, 0, 0] = below * math.log(2) * math.sqrt(d) / 4
    k[:, :, 1:, 1] = torch.randn(n - 1, generator=g, device="cuda")
    v[:, :, 0] = 2.0 ** -20
    q, k, v = (t.to(DT[dtype]) for t in (q, k, v))
    out, lse = torch.empty_like(q), torch.empty(1, 1, n, device="cuda")
    B.d2o_prompt_attention(q, k, v, out, lse=lse)
    i = torch.tensor([1, 100, 5000, n - 1], device="cuda")
    Q, K, V = q[0, 0, i].double(), k[0, 0].double(), v[0, 0].double()
    x = (Q @ K.T / math.sqrt(d)).masked_fill(torch.arange(n, device="cuda")[None] > i[:, None], -math.inf)
    p = torch.softmax(x, 1)
    delta = 16 * 2.0 ** -24 * float((Q.abs() @ K.abs().T).max()) / math.sqrt(d)
    e = ((0.0 if dtype == "f32" else torch.finfo(DT[dtype]).eps / 2) + 2 * delta + 2.0 ** -21) * (p @ V.abs())
    if dtype == "f16":
        e += 2.0 ** -32 * ((p > 0) * (p < 2.0 ** -21 * p.amax(1, keepdim=True))).double() @ V.abs() * p.amax(1, keepdim=True)
    ref, o = p @ V, out[0, 0, i].double()
    assert bool((((ref - e).to(DT[dtype]).double() <= o) & (o <= (ref + e).to(DT[dtype]).double())).all()), ((o - ref) / ref).abs().amax(1).tolist()
    y = torch.logsumexp(x, 1)
    assert bool(((lse[0, 0, i].double() - y).abs() <= delta + 2.0 ** -22 * y.abs().clamp(min=1)).all())


@pytest.mark.parametrize("dtype,scale", [("f16", 1000), ("f16", 8000), ("f16", 30000), ("bf16", 1000), ("bf16", 5e4), ("bf16", 1e9), ("bf16", 1e17), ("f32", 1e8)])
@pytest.mark.parametrize("d,window,sinks", [(128, 0, 0), (64, 0, 0), (128, 100, 3)])
def test_huge_logits(cuda_device, dtype, scale, d, window, sinks):
    """Logits up to the largest that fp32 sums hold: a row is the value of its largest logit wherever that leads the next by more than the
    logits' own error (2 delta of the tolerance) and by 40, and never NaN; beside them rows of ordinary size."""
    n = 500
    q, k, v = draw(n, 1, 2, 1, n, d, "f32")
    limit = torch.finfo(DT[dtype]).max
    q, k, v = ((t * scale).clamp(-limit, limit).to(DT[dtype]) for t in (q, k, v / scale))
    q[:, :, ::7] = (q[:, :, ::7].float() / (float(scale) * scale)).to(DT[dtype])                       # logits of a few units
    out, lse = torch.full_like(q, float("nan")), torch.empty(1, 2, n, device="cuda")
    B.d2o_prompt_attention(q, k, v, out, lse=lse, window=window, n_sink=sinks)
    assert bool(torch.isfinite(out.float()).all()) and bool(torch.isfinite(lse).all())
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    seen = (j <= i) & ((j > i - window) | (j < sinks)) if window > 0 else j <= i
    K, V = k[0, 0].double(), v[0, 0].double()
    for h in range(2):
        Q = q[0, h].double()
        x = (Q @ K.T / math.sqrt(d)).masked_fill(~seen, -math.inf)
        delta = 16 * 2.0 ** -24 * (Q.abs() @ K.abs().T / math.sqrt(d)).masked_fill(~seen, 0).amax(1)
        two = x.topk(2, dim=1).values
        clear = (two[:, 0] - two[:, 1] > 2 * delta + 40) | (torch.arange(n, device="cuda") == 0)
        assert int(clear.sum()) > (300 if scale > 500 else 0)
        # one weight of nearly 1: it is off by its own rounding against the sum, and the division by 2^-21
        weights = 0.0 if dtype == "f32" else torch.finfo(DT[dtype]).eps / 2
        one, o = V[x.argmax(1)][clear], out[0, h][clear].double()
        e = (weights + 2.0 ** -21) * one.abs()
        assert bool((((one - e).to(DT[dtype]).double() <= o) & (o <= (one + e).to(DT[dtype]).double())).all())
        assert bool(((lse[0, h].double() - torch.logsumexp(x, 1)).abs()[clear] <= (delta + 2.0 ** -22 * two[:, 0].abs().clamp(min=1))[clear]).all())
        small = torch.arange(0, n, 7, device="cuda")
        p = torch.softmax(x[small], 1)
        e = (weights + 2 * delta[small, None] + 2.0 ** -21) * (p @ V.abs())
        ref, o = p @ V, out[0, h][small].double()
        assert bool((((ref - e).to(DT[dtype]).double() <= o) & (o <= (ref + e).to(DT[dtype]).double())).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_huge_logits_come_and_go(cuda_device, dtype, d):
    """References of -5e6 that give way to ordinary logits at key 200, and one key of +5e6 at 350: rows 200 .. 349 are those of a prompt without
    the first 200 keys (delta from theirs alone), rows from 350 on are that key's value (see test_huge_logits)."""
    n = 700
    q, k, v = draw(21, 1, 1, 1, n, d, "f32")
    q, k = q * 0.5, k * 0.5
    q[..., 0], k[..., 0] = 8000.0, 0.0
    k[:, :, :200, 0], k[:, :, 350, 0] = -8000.0, 8000.0
    q, k, v = (t.to(DT[dtype]) for t in (q, k, v))
    out, lse = torch.full_like(q, float("nan")), torch.empty(1, 1, n, device="cuda")
    B.d2o_prompt_attention(q, k, v, out, lse=lse)
    assert bool(torch.isfinite(out.float()).all()) and bool(torch.isfinite(lse).all())
    check(q[0, 0, 200:350], k[0, 0, 200:350], v[0, 0, 200:350], out[0, 0, 200:350], lse[0, 0, 200:350], 0, 0, dtype)
    weights = 0.0 if dtype == "f32" else torch.finfo(DT[dtype]).eps / 2
    one, o = v[0, 0, 350].double(), out[0, 0, 350:].double()
    e = (weights + 2.0 ** -21) * one.abs()
    assert bool((((one - e).to(DT[dtype]).double() <= o) & (o <= (one + e).to(DT[dtype]).double())).all())


def test_not_finite(cuda_device):
    """A NaN key reaches the rows that see it and no others; +inf and -inf logits give NaN and 0 as the formula does."""
    for dtype in DT:
        q, k, v = draw(9, 1, 1, 1, 600, 64, dtype)
        q[0, 0, :, 0] = 1.0
        k[0, 0, :, 0] = 0.0
        k[0, 0, 300, 0], k[0, 0, 500, 0] = float("-inf"), float("nan")
        out, lse = torch.empty_like(q), torch.empty(1, 1, 600, device="cuda")
        B.d2o_prompt_attention(q, k, v, out, lse=lse)
        assert bool(torch.isfinite(out[0, 0, :500].float()).all()) and bool(out[0, 0, 500:].isnan().all()) and bool(lse[0, 0, 500:].isnan().all())
        keep = torch.tensor([j for j in range(500) if j != 300], device="cuda")
        # rows behind 300 are those of a prompt without that key
        ref, ref_lse, _, _ = reference(q[0, 0][keep], k[0, 0][keep], v[0, 0][keep], 0, 0)
        assert float((lse[0, 0][keep].double() - ref_lse).abs().max()) < 2e-5
        k[0, 0, 500, 0] = float("inf")
        B.d2o_prompt_attention(q, k, v, out, lse=lse)
        assert bool(torch.isfinite(out[0, 0, :500].float()).all()) and bool(out[0, 0, 500:].isnan().all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,window,sinks,at", [(1000, 200, 0, 0), (1000, 200, 0, 56), (1000, 200, 4, 4), (1000, 200, 4, 50), (1500, 130, 200, 200), (1500, 130, 200, 255),
                                               (900, 64, 0, 300), (900, 300, 3, 700), (700, 0, 0, 600), (2000, 257, 129, 511), (800, 1, 0, 255), (1300, 128, 5, 127)])
def test_values_that_are_not_finite(cuda_device, dtype, d, n, window, sinks, at):
    """An infinite or NaN value reaches the rows that see its key, and of the others those in a block of 256 queries of which one sees it at most; a
    key that is not finite the rows that see it alone."""
    q, k, v = draw(n + at, 1, 2, 1, n, d, dtype)
    want, out = torch.empty_like(q), torch.empty_like(q)
    B.d2o_prompt_attention(q, k, v, want, window=window, n_sink=sinks)
    i = torch.arange(n, device="cuda")
    sees = (i >= at) & ((i < at + window) | (at < sinks)) if window else i >= at
    blocks = torch.zeros(-(-n // 256), dtype=torch.bool, device="cuda")
    blocks[i[sees] // 256] = True
    apart = ~blocks[i // 256]
    for bad in (math.inf, -math.inf, math.nan):
        x = v.clone()
        x[0, 0, at] = bad
        B.d2o_prompt_attention(q, k, x, out, window=window, n_sink=sinks)
        assert bool((~torch.isfinite(out[:, :, sees].float())).all())
        assert torch.equal(out[:, :, apart], want[:, :, apart])
        x = k.clone()
        x[0, 0, at] = math.nan
        B.d2o_prompt_attention(q, x, v, out, window=window, n_sink=sinks)
        assert bool(out[:, :, sees].isnan().all()) and torch.equal(out[:, :, ~sees], want[:, :, ~sees])


def test_normalisers_feed_the_column_sums(cuda_device):
    """lse as d2o_layer_stats takes it: the same column sums, to rounding, as with its own first sweep."""
    q, k, v = draw(3, 1, 8, 2, 777, 128, "bf16")
    sums = []
    for given in (False, True):
        ctx = B.D2OContext(B.make_config(n_layers=1, batch=1, n_q_heads=8, n_kv_heads=2, d_head=128, dtype="bf16", prompt_len=777,
                                         max_new_tokens=1, rho=0.5))
        lse, out = torch.empty(1, 8, 777, device="cuda"), torch.empty_like(q)
        if given:
            B.d2o_prompt_attention(q, k, v, out, lse=lse)
        ctx.d2o_layer_stats(0, q, k, lse if given else None)
        sums.append(ctx.colsum(0).clone())
        ctx.close()
    torch.testing.assert_close(sums[0], sums[1], rtol=2e-5, atol=1e-7)


@pytest.mark.parametrize("dtype,d,hq", [("bf16", 128, 17), ("f16", 64, 34), ("f32", 128, 17)])
def test_longest_prompt_and_offsets_past_32_bits(cuda_device, dtype, d, hq):
    """2^20 tokens under a window, more than 2^31 elements of queries: rows of the first and of the last head."""
    n, window, sinks = 1 << 20, 300, 5
    g = torch.Generator(device="cuda").manual_seed(hq)
    q, k, v = (torch.empty(1, h, n, d, dtype=DT[dtype], device="cuda").normal_(generator=g) for h in (hq, 1, 1))
    out, lse = torch.full_like(q, float("nan")), torch.full((1, hq, n), float("nan"), device="cuda")
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    B.d2o_prompt_attention(q, k, v, out, lse=lse, window=window, n_sink=sinks, status=status)
    assert status.tolist() == [0, 0]
    for h in (0, hq - 1):
        for end in (600, n // 2 + 77, n):
            a = end - 600
            cols = torch.cat([torch.arange(min(sinks, max(0, a - window)), device="cuda"), torch.arange(max(0, a - window), end, device="cuda")])
            K, V = k[0, 0, cols], v[0, 0, cols]
            rows = torch.arange(a, end, device="cuda")
            i, j = rows[:, None], cols[None]
            seen = (j <= i) & ((j > i - window) | (j < sinks))
            Q = q[0, h, rows].double()
            x = (Q @ K.double().T / math.sqrt(d)).masked_fill(~seen, -math.inf)
            y = torch.logsumexp(x, 1)
            p = torch.exp(x - y[:, None])
            delta = 16 * 2.0 ** -24 * float((Q.abs() @ K.double().abs().T).max()) / math.sqrt(d)
            weights = 0.0 if dtype == "f32" else torch.finfo(DT[dtype]).eps / 2
            e, ref, o = (weights + 2 * delta + 2.0 ** -21) * (p @ V.double().abs()), p @ V.double(), out[0, h, rows].double()
            assert bool((((ref - e).to(DT[dtype]).double() <= o) & (o <= (ref + e).to(DT[dtype]).double())).all()), (h, end)
            assert bool(((lse[0, h, rows].double() - y).abs() <= delta + 2.0 ** -22 * y.abs().clamp(min=1)).all())
    assert not bool(lse.isnan().any()) and not any(bool(out[0, h].isnan().any()) for h in range(hq))


def test_streams_graph_and_repeats(cuda_device):
    """On a stream other than the default one, captured and replayed with other inputs, the same bits every time."""
    q, k, v = draw(11, 2, 4, 2, 385, 128, "f16")
    want = torch.empty_like(q)
    B.d2o_prompt_attention(q, k, v, want, window=100, n_sink=2)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out, q2 = torch.zeros_like(q), torch.zeros_like(q)
    with torch.cuda.stream(s):
        B.d2o_prompt_attention(q2, k, v, out, window=100, n_sink=2)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        B.d2o_prompt_attention(q2, k, v, out, window=100, n_sink=2)
    for _ in range(3):
        q2.copy_(q)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
