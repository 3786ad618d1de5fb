"""A cache in pages (d2o_paged_append, d2o_paged_decode_step, d2o_paged_evict) against plain statements of the formulas in
float64 on the host, and the three in a row as a serving program uses them.

Every test compares whole pools: what a call does not own must keep its bits, and all of it holds NaN at first, so that a row
read where nothing was put shows.  Rows and positions are compared exactly.

Tolerance of the attention.  A logit errs by a few 2^-24 of the magnitudes that it sums: delta = 16 * 2^-24 * max_j sum_e |q_e
k_je| / sqrt(d).  A weight is off by a factor of at most 1 + 2 delta (itself, the sum), and by 2^-20 from exp2, the joins and, for
16-bit caches, the two 16-bit terms in which it enters the products (bf16: 2^-16 more).  An output is the rounding of something
within e = (2 delta + 2^-20 + 2^-16) * sum_j p_j |v_j| of the reference (fp32 and fp16: without 2^-16); a score is off by 2 delta +
2^-20 of the added weight, and by the rounding of the sum."""
import math

import numpy as np
import pytest
import torch

from paper_2406_13035_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NAN = float("nan")


def bits(t):
    return t.detach().cpu().contiguous().view({4: torch.int32, 2: torch.int16}[t.element_size()]).numpy()


class Paged:
    """A cache, its pools full of NaN, with `spare` pages that no table names; a host copy of what should be in it."""

    def __init__(self, seed, b, hq, hkv, d, dtype, page, max_pages, lens, scored=True, spare=2):
        self.g = torch.Generator().manual_seed(seed)
        self.b, self.hq, self.hkv, self.d, self.page, self.dt, self.dtype = b, hq, hkv, d, page, DT[dtype], dtype
        n_pages = b * max_pages + spare
        self.table = torch.randperm(n_pages, generator=self.g)[: b * max_pages].view(b, max_pages).to(torch.int32)
        self.len = torch.as_tensor(lens, dtype=torch.int32)
        if self.len.dim() == 1:
            self.len = self.len[:, None].expand(b, hkv).contiguous()
        shape = (n_pages, hkv, page)
        self.k, self.v = torch.full((*shape, d), NAN, dtype=self.dt), torch.full((*shape, d), NAN, dtype=self.dt)
        self.pos = torch.full(shape, -7, dtype=torch.int32) if scored else None
        self.score = torch.full(shape, NAN) if scored else None
        reach = max_pages * page
        for i in range(b):
            for h in range(hkv):
                for r in range(min(int(self.len[i, h]), reach)):
                    pg, at = self.at(i, r)
                    self.k[pg, h, at] = torch.randn(d, generator=self.g).to(self.dt)
                    self.v[pg, h, at] = torch.randn(d, generator=self.g).to(self.dt)
                    if scored:
                        self.pos[pg, h, at], self.score[pg, h, at] = r, float(torch.rand(1, generator=self.g))
        self.upload()

    def upload(self):
        dev = lambda t: None if t is None else t.cuda()
        self.dk, self.dv, self.dpos, self.dscore, self.dtable, self.dlen = map(dev, (self.k, self.v, self.pos, self.score, self.table, self.len))
        self.cache = B.D2OPagedCache(self.dk, self.dv, self.dtable, self.dlen, n_q_heads=self.hq, pos=self.dpos, score=self.dscore)

    def at(self, i, r):
        return int(self.table[i, r // self.page]), r % self.page

    def randn(self, *s):
        return torch.randn(*s, generator=self.g).to(self.dt)

    def rows(self, pool, i, h, rs):
        return torch.stack([pool[self.at(i, r)[0], h, self.at(i, r)[1]] for r in rs]) if len(rs) else pool.new_zeros(0, *pool.shape[3:])

    def same(self, scores=True):
        """The device's pools are the host's, bit for bit."""
        for name, host, dev in (("k", self.k, self.dk), ("v", self.v, self.dv), ("pos", self.pos, self.dpos), ("score", self.score, self.dscore)):
            if host is not None and (scores or name != "score"):
                assert np.array_equal(bits(host), bits(dev)), name
        assert torch.equal(self.len, self.dlen.cpu()) and torch.equal(self.table, self.dtable.cpu())

    # ---- the plain statements
    def append(self, K, V, lens=None, first=None, colsum=None):
        n = K.shape[2]
        for i in range(self.b):
            for h in range(self.hkv):
                for j in range(min(n, n if lens is None else int(lens[i])) if self.len[i, h] >= 0 else 0):
                    pg, at = self.at(i, int(self.len[i, h]) + j)
                    self.k[pg, h, at], self.v[pg, h, at] = K[i, h, j], V[i, h, j]
                    if self.pos is not None:
                        self.pos[pg, h, at] = (0 if first is None else int(first[i])) + j
                        s = torch.zeros(())
                        if colsum is not None:
                            G = self.hq // self.hkv
                            s = colsum[i, h * G, j]
                            for g in range(1, G):
                                s = s + colsum[i, h * G + g, j]
                        self.score[pg, h, at] = s

    def step(self, q, k, v, out, positions, window, n_sink):
        """Checks `out` and the device's scores, and takes the scores over (they are sums of rounded terms)."""
        G = self.hq // self.hkv
        got_scores = None if self.score is None else self.dscore.cpu()
        for i in range(self.b):
            for h in range(self.hkv):
                t = int(self.len[i, h])
                if t < 0:
                    assert bool((out[i, h * G:(h + 1) * G] == 3).all())
                    continue
                pg, at = self.at(i, t)
                self.k[pg, h, at], self.v[pg, h, at] = k[i, h], v[i, h]
                rs = [r for r in range(t + 1) if window == 0 or r > t - window or r < n_sink]
                K, V = self.rows(self.k, i, h, rs).double(), self.rows(self.v, i, h, rs).double()
                Q = q[i, h * G:(h + 1) * G].double()
                p = torch.softmax(Q @ K.T / math.sqrt(self.d), -1)
                delta = 16 * 2.0 ** -24 * float((Q.abs() @ K.abs().T).max()) / math.sqrt(self.d)
                w = 2 * delta + 2.0 ** -20
                ref, e = p @ V, (w + (2.0 ** -16 if self.dtype == "bf16" else 0)) * (p @ V.abs())
                o = out[i, h * G:(h + 1) * G].cpu().double()
                ok = ((ref - e).to(self.dt).double() <= o) & (o <= (ref + e).to(self.dt).double())
                assert bool(ok.all()), (i, h, float(((o - ref).abs() / e).max()))
                if self.score is not None:
                    self.pos[pg, h, at] = t if positions is None else int(positions[i])
                    add = p.sum(0)
                    for r, x in zip(rs, add.tolist()):
                        pr, ar = self.at(i, r)
                        was = 0.0 if r == t else float(self.score[pr, h, ar])
                        now = float(got_scores[pr, h, ar])
                        assert abs(now - (was + x)) <= w * x + 2.0 ** -24 * abs(was + x), (i, h, r)
                        self.score[pr, h, ar] = now

    def evict(self, budgets, next_pos, n_sink, window):
        for i in range(self.b):
            for h in range(self.hkv):
                n, s = int(self.len[i, h]), int(budgets[i, h])
                if n < 0 or n <= s or s < 0:
                    continue
                pos = self.rows(self.pos, i, h, range(n)).tolist()
                score = self.rows(self.score, i, h, range(n)).tolist()

                def rank(r):
                    protected = pos[r] < n_sink or pos[r] >= int(next_pos[i]) - window
                    nan = score[r] != score[r]
                    return (not protected, protected is False and not nan, 0 if protected or nan else -score[r], pos[r])
                kept = sorted(sorted(range(n), key=rank)[:s])
                holes = [r for r in range(s) if r not in set(kept)]
                movers = [r for r in kept if r >= s]
                assert len(holes) == len(movers)
                for to, frm in zip(holes, movers):
                    (tp, ta), (fp, fa) = self.at(i, to), self.at(i, frm)
                    for pool in (self.k, self.v, self.pos, self.score):
                        pool[tp, h, ta] = pool[fp, h, fa]


# ---------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("b,hq,hkv,d,dtype,page,n,lens,held,scored", [
    (1, 1, 1, 64, "f32", 16, 1, None, [0], True), (2, 4, 2, 128, "bf16", 16, 5, [5, 0], [15, 16], True),
    (3, 8, 2, 128, "f16", 32, 70, [70, 33, 1], [0, 31, 7], True), (2, 2, 2, 64, "bf16", 64, 130, None, [63, -1], False),
    (2, 16, 2, 128, "f32", 16, 65, [200, 64], [1, 2], True), (1, 3, 3, 64, "f16", 1024, 64, [-3], [5], False)])
def test_append(cuda_device, b, hq, hkv, d, dtype, page, n, lens, held, scored):
    c = Paged(n, b, hq, hkv, d, dtype, page, (n + max(held) + page - 1) // page + 1, held, scored)
    K, V = c.randn(b, hkv, n, d), c.randn(b, hkv, n, d)
    first = torch.arange(b, dtype=torch.int32) * 1000 + 5 if scored else None
    colsum = torch.rand(b, hq, n, generator=c.g) if scored else None
    up = lambda t: None if t is None else t.cuda()
    li = None if lens is None else torch.tensor(lens, dtype=torch.int32)
    c.cache.d2o_paged_append(K.cuda(), V.cuda(), lens=up(li), first_pos=up(first), colsum=up(colsum))
    c.append(K, V, li, first, colsum)
    c.same()
    if scored:                                                                 # defaults: positions from 0, scores 0
        c.cache.d2o_paged_append(K.cuda(), V.cuda(), lens=up(li))
        c.append(K, V, li)
        c.same()
    c.cache.check()


# ---------------------------------------------------------------------------------------------- decode
STEPS = [  # batch, q heads, kv heads, d, page, rows held, window, sinks, scores
    (1, 1, 1, 64, 16, [0], 0, 0, True), (1, 2, 1, 128, 16, [1], 0, 0, True), (2, 4, 1, 128, 16, [15, 16], 0, 0, True),
    (3, 8, 1, 64, 32, [17, 31, 47], 0, 0, True), (2, 8, 2, 128, 64, [300, 3], 0, 0, True), (1, 4, 4, 64, 1024, [700], 0, 0, False),
    (4, 4, 2, 128, 16, [100, -1, 0, 255], 0, 0, True), (2, 2, 2, 128, 16, [200, 90], 1, 0, True), (2, 2, 1, 64, 16, [200, 90], 33, 0, True),
    (3, 4, 2, 128, 32, [500, 40, 64], 64, 4, True), (2, 8, 1, 128, 16, [600, 100], 100, 17, True), (1, 4, 1, 64, 128, [900], 500, 300, True),
    (1, 4, 1, 128, 16, [64], 1000, 4, False), (1, 16, 2, 128, 64, [1700], 0, 0, True), (40, 4, 4, 64, 16, list(range(0, 120, 3)), 0, 0, True),
    (300, 2, 1, 64, 16, [7] * 299 + [333], 0, 0, False)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("b,hq,hkv,d,page,held,window,sinks,scored", STEPS)
def test_decode_step(cuda_device, b, hq, hkv, d, page, held, window, sinks, scored, dtype):
    """Two steps in a row, the lengths advanced in between as the caller does."""
    c = Paged(sum(held) + window, b, hq, hkv, d, dtype, page, (max(held) + 2 + page - 1) // page, held, scored)
    for step in range(2):
        q, k, v = c.randn(b, hq, d), c.randn(b, hkv, d), c.randn(b, hkv, d)
        positions = torch.arange(b, dtype=torch.int32) + 9000 if scored and step else None
        out = torch.full((b, hq, d), 3.0, dtype=c.dt, device="cuda")
        c.cache.d2o_paged_decode_step(q.cuda(), k.cuda(), v.cuda(), out, positions=None if positions is None else positions.cuda(),
                                      window=window, n_sink=sinks)
        c.step(q, k, v, out, positions, window, sinks)
        c.same()
        c.cache.check()
        c.len += (c.len >= 0).to(torch.int32)
        c.dlen.copy_(c.len)


def test_decode_heads_of_different_lengths(cuda_device):
    c = Paged(1, 2, 4, 2, 128, "bf16", 16, 8, [[5, 90], [33, -1]])
    q, k, v = c.randn(2, 4, 128), c.randn(2, 2, 128), c.randn(2, 2, 128)
    out = torch.full((2, 4, 128), 3.0, dtype=c.dt, device="cuda")
    c.cache.d2o_paged_decode_step(q.cuda(), k.cuda(), v.cuda(), out)
    c.step(q, k, v, out, None, 0, 0)
    c.same()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decode_shared_prefix(cuda_device, dtype):
    """Two sequences with the same first pages, without scores."""
    c = Paged(2, 2, 4, 2, 64, dtype, 16, 6, [70, 83], scored=False)
    for r in range(48):
        for h in range(2):
            for pool in (c.k, c.v):
                pool[c.at(1, r)[0], h, c.at(1, r)[1]] = NAN
    c.table[1, :3] = c.table[0, :3]
    c.upload()
    q, k, v = c.randn(2, 4, 64), c.randn(2, 2, 64), c.randn(2, 2, 64)
    out = torch.full((2, 4, 64), 3.0, dtype=c.dt, device="cuda")
    c.cache.d2o_paged_decode_step(q.cuda(), k.cuda(), v.cuda(), out)
    c.step(q, k, v, out, None, 0, 0)
    c.same()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_decode_long(cuda_device, dtype):
    """40000 rows over every SM, made and checked on the GPU: logits of variance 1, so that every row counts."""
    n, page, d, hkv, G = 40000, 64, 128, 2, 4
    g = torch.Generator(device="cuda").manual_seed(1)
    per = (n + page) // page
    table = torch.randperm(per + 1, generator=g, device="cuda")[:per].to(torch.int32)[None].contiguous()
    kp, vp = (torch.randn(per + 1, hkv, page, d, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    pos, score = torch.zeros(per + 1, hkv, page, dtype=torch.int32, device="cuda"), torch.zeros(per + 1, hkv, page, device="cuda")
    length = torch.full((1, hkv), n, dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(1, h, d, generator=g, device="cuda").to(DT[dtype]) for h in (hkv * G, hkv, hkv))
    out = torch.empty_like(q)
    c = B.D2OPagedCache(kp, vp, table, length, n_q_heads=hkv * G, pos=pos, score=score)
    c.d2o_paged_decode_step(q, k, v, out)
    again = torch.empty_like(q)
    first = score.clone()
    c.d2o_paged_decode_step(q, k, v, again)
    assert torch.equal(out, again)
    for h in range(hkv):
        rows = lambda pool: pool[table[0].long()].transpose(0, 1).flatten(1, 2)[h, :n + 1].double()
        K, V, Q = rows(kp), rows(vp), q[0, h * G:(h + 1) * G].double()
        assert torch.equal(K[n], k[0, h].double()) and torch.equal(V[n], v[0, h].double())
        p = torch.softmax(Q @ K.T / math.sqrt(d), -1)
        w = 32 * 2.0 ** -24 * float((Q.abs() @ K.abs().T).max()) / math.sqrt(d) + 2.0 ** -20
        e = (w + (2.0 ** -16 if dtype == "bf16" else 0)) * (p @ V.abs())
        ref, o = p @ V, out[0, h * G:(h + 1) * G].double()
        assert bool((((ref - e).to(DT[dtype]).double() <= o) & (o <= (ref + e).to(DT[dtype]).double())).all())
        s = first[table[0].long()].transpose(0, 1).flatten(1, 2)[h, :n + 1].double()
        assert bool(((s - p.sum(0)).abs() <= (w + 2.0 ** -24) * p.sum(0)).all())
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,G,room", [(64, 1, 0), (128, 4, 0), (128, 2, 40000)])
@pytest.mark.parametrize("below", [14, 18, 22.3, 27, 31])
def test_decode_many_small_weights_beside_a_large_one(cuda_device, dtype, d, G, room, below):
    """One row with nearly all of the weight and a value of nearly zero, and 8000 rows at 2^-below of it with values of one sign: what the small weights
    lose in their rounding does not average out.  Beyond the tolerance of the other tests an fp16 weight below 2^-16 of the row's largest is off by
    2^-39 of it (the largest is 2^14; the second term's half step is 2^-25 where it is subnormal), and the fp32 sum over the rows of a warp grows by
    one product of 16 rows, of two terms each, at a time, each off by up to a unit in its last place (2^-23; 8000 rows over at least eight warps: 63 products)."""
    n, page = 8000, 16
    g = torch.Generator(device="cuda").manual_seed(5)
    per = n // page + 1
    table = torch.full((1, max(per, room // page)), -1, dtype=torch.int32, device="cuda")
    table[0, :per] = torch.randperm(per, generator=g, device="cuda")
    K = torch.zeros(per * page, d, device="cuda")
    V = 4 + torch.rand(per * page, d, generator=g, device="cuda")
    K[0, 0], V[0] = below * math.log(2) * math.sqrt(d) / 4, 2.0 ** -20
    K[1:, 1] = torch.randn(per * page - 1, generator=g, device="cuda")
    q = torch.zeros(1, G, d, device="cuda")
    q[..., 0] = 4.0
    K, V, q = (t.to(DT[dtype]) for t in (K, V, q))
    kp, vp = (torch.empty(per, 1, page, d, dtype=DT[dtype], device="cuda") for _ in range(2))
    kp[table[0, :per].long()], vp[table[0, :per].long()] = K.view(per, 1, page, d), V.view(per, 1, page, d)
    pos, score = torch.zeros(per, 1, page, dtype=torch.int32, device="cuda"), torch.zeros(per, 1, page, device="cuda")
    c = B.D2OPagedCache(kp, vp, table, torch.full((1, 1), n - 1, dtype=torch.int32, device="cuda"), n_q_heads=G, pos=pos, score=score)
    out = torch.empty_like(q)
    c.d2o_paged_decode_step(q, K[None, None, n - 1].contiguous(), V[None, None, n - 1].contiguous(), out)
    c.check()
    Q, Kd, Vd = q[0].double(), K[:n].double(), V[:n].double()
    x = Q @ Kd.T / math.sqrt(d)
    p = torch.softmax(x, 1)
    delta = 16 * 2.0 ** -24 * float((Q.abs() @ Kd.abs().T).max()) / math.sqrt(d)
    w = 2 * delta + 2.0 ** -20
    mag = p @ Vd.abs()
    e = (w + (2.0 ** -16 if dtype == "bf16" else 0) + 2 * 63 * 2.0 ** -23) * mag
    if dtype == "f16":
        e += 2.0 ** -39 * p.amax(1, keepdim=True) * ((p < 2.0 ** -16 * p.amax(1, keepdim=True)).double() @ Vd.abs())
    ref, o = p @ Vd, out[0].double()
    assert bool((((ref - e).to(DT[dtype]).double() <= o) & (o <= (ref + e).to(DT[dtype]).double())).all()), ((o - ref) / ref).abs().amax().item()
    got = score[table[0, :per].long()].flatten()[:n].double()
    assert bool(((got - p.sum(0)).abs() <= (w + 2.0 ** -24) * p.sum(0)).all())


@pytest.mark.parametrize("dtype,scale", [("f32", 1e9), ("f16", 300), ("f16", 3000), ("f16", 12000), ("f16", 30000), ("bf16", 3000), ("bf16", 1e9), ("bf16", 1e17)])
@pytest.mark.parametrize("d,G", [(64, 1), (128, 4)])
def test_decode_huge_logits(cuda_device, dtype, scale, d, G):
    """Logits up to the largest that fp32 sums hold: the value of the row with the largest, exactly, where that leads the next by more than the
    logits' own error and by 100, so that every other weight is zero beside it."""
    c = Paged(31, 1, G, 1, d, dtype, 16, 20, [300], scored=False)
    limit = torch.finfo(DT[dtype]).max
    big = lambda t: (t.float() * scale).clamp(-limit, limit).to(DT[dtype])
    c.k.copy_(big(c.k))
    c.upload()
    q, k, v = big(c.randn(1, G, d)), big(c.randn(1, 1, d)), c.randn(1, 1, d)
    out = torch.full((1, G, d), 3.0, dtype=c.dt, device="cuda")
    c.cache.d2o_paged_decode_step(q.cuda(), k.cuda(), v.cuda(), out)
    K = torch.cat([c.rows(c.k, 0, 0, range(300)), k[0]]).double()
    V = torch.cat([c.rows(c.v, 0, 0, range(300)), v[0]])
    Q = q[0].double()
    x = Q @ K.T / math.sqrt(d)
    delta = 16 * 2.0 ** -24 * (Q.abs() @ K.abs().T / math.sqrt(d)).amax(1)
    two = x.topk(2, dim=1).values
    clear = two[:, 0] - two[:, 1] > 2 * delta + 100
    assert bool(clear.any()) and torch.equal(out[0].cpu()[clear], V[x.argmax(1)][clear]) and bool(torch.isfinite(out.float()).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,G", [(64, 1), (128, 4), (64, 8), (128, 2)])
@pytest.mark.parametrize("n,room", [(5, 16), (300, 320), (2000, 2016), (2000, 60000)])
def test_decode_rows_that_are_not_finite(cuda_device, dtype, d, G, n, room):
    """Rows that are seen: infinite values give infinities, of both signs or NaN ones NaN, in those elements alone; a logit of -inf a weight of zero, a
    NaN one NaN in the heads of its slice.  Weights are within 2^-20 of the largest."""
    page, hkv = 16, 3
    g = torch.Generator(device="cuda").manual_seed(n + d + G)
    per = n // page + 1
    table = torch.full((1, room // page + 1), -1, dtype=torch.int32, device="cuda")
    table[0, :per] = torch.randperm(per, generator=g, device="cuda")
    at = lambda r: (int(table[0, r // page]), r % page)
    kp, vp = (torch.randn(per, hkv, page, d, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    q, k, v = (torch.randn(1, h, d, generator=g, device="cuda").to(DT[dtype]) for h in (hkv * G, hkv, hkv))
    kp[..., 5], k[..., 5], q[..., 5] = 0.0, 0.0, 1.0
    pos, score = torch.zeros(per, hkv, page, dtype=torch.int32, device="cuda"), torch.zeros(per, hkv, page, device="cuda")
    c = B.D2OPagedCache(kp, vp, table, torch.full((1, hkv), n, dtype=torch.int32, device="cuda"), n_q_heads=hkv * G, pos=pos, score=score)
    want, out = torch.empty_like(q), torch.empty_like(q)
    c.d2o_paged_decode_step(q, k, v, want)
    rows = [0, n // 3, n - 1]
    for r, e, x in [(rows[0], 1, math.inf), (rows[1], 2, -math.inf), (rows[2], 3, math.nan), (rows[0], 4, math.inf), (rows[2], 4, -math.inf), (rows[1], 9, math.inf), (rows[2], 9, math.inf)]:
        vp[at(r)[0], 0, at(r)[1], e] = x
    vn = v.clone()
    vn[0, 0, 7] = -math.inf                                                    # the new token's own
    kp[at(rows[1])[0], 1, at(rows[1])[1], 5] = -math.inf
    kp[at(rows[2])[0], 2, at(rows[2])[1], 5] = math.nan
    score.zero_()
    c.d2o_paged_decode_step(q, k, vn, out)
    c.check()
    o = out[0].view(hkv, G, d)
    first = o[0].float()
    assert bool((first[:, [1, 9]] == math.inf).all()) and bool((first[:, [2, 7]] == -math.inf).all()) and bool(first[:, [3, 4]].isnan().all())
    rest = [e for e in range(d) if e not in (1, 2, 3, 4, 7, 9)]
    assert torch.equal(first[:, rest], want[0].view(hkv, G, d)[0].float()[:, rest])
    assert bool(o[2].isnan().all())
    # slice 1: as without that row
    keep = [r for r in range(n) if r != rows[1]]
    line = lambda pool, h: pool[table[0, :per].long(), h].flatten(0, 1)
    K, V, Q = torch.cat([line(kp, 1)[keep], k[0, 1:2]]).double(), torch.cat([line(vp, 1)[keep], v[0, 1:2]]).double(), q[0, G:2 * G].double()
    p = torch.softmax(Q @ K.T / math.sqrt(d), -1)
    w = 32 * 2.0 ** -24 * float((Q.abs() @ K.abs().T).max()) / math.sqrt(d) + 2.0 ** -20
    e, ref = (w + (2.0 ** -16 if dtype == "bf16" else 0)) * (p @ V.abs()), p @ V
    assert bool((((ref - e).to(DT[dtype]).double() <= o[1].double()) & (o[1].double() <= (ref + e).to(DT[dtype]).double())).all())
    assert float(score[at(rows[1])[0], 1, at(rows[1])[1]]) == 0.0
    assert bool((line(score, 1)[:n + 1][keep] > 0).all()) and bool(line(score, 2)[:n + 1].isnan().all()) and bool(torch.isfinite(line(score, 0)[:n + 1]).all())


def test_decode_offsets_past_32_bits(cuda_device):
    """A pool of more than 2^31 elements, and rows of it behind that border."""
    page, d, hkv, dt = 1024, 128, 8, torch.bfloat16
    n_pages = (1 << 31) // (page * d * hkv) + 8
    kp = torch.zeros(n_pages, hkv, page, d, dtype=dt, device="cuda")
    vp = torch.zeros_like(kp)
    g = torch.Generator(device="cuda").manual_seed(3)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 3]], dtype=torch.int32, device="cuda")
    for p in table[0].tolist():
        kp[p], vp[p] = (torch.randn(hkv, page, d, generator=g, device="cuda").to(dt) for _ in range(2))
    n = 2 * page + 100
    length = torch.full((1, hkv), n, dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(1, hkv, d, generator=g, device="cuda").to(dt) for _ in range(3))
    out = torch.empty_like(q)
    c = B.D2OPagedCache(kp, vp, table, length, n_q_heads=hkv)
    c.d2o_paged_decode_step(q, k, v, out)
    K, V = (pool[table[0].long()].transpose(0, 1).flatten(1, 2)[:, :n + 1].double() for pool in (kp, vp))
    assert torch.equal(K[:, n], k[0].double()) and torch.equal(V[:, n], v[0].double())
    p = torch.softmax(torch.einsum("hd,hnd->hn", q[0].double(), K) / math.sqrt(d), -1)
    torch.testing.assert_close(out[0].double(), torch.einsum("hn,hnd->hd", p, V), rtol=2.0 ** -8, atol=1e-5)
    more = torch.randn(1, hkv, 5, d, generator=g, device="cuda").to(dt)
    c.d2o_paged_append(more, more)
    assert torch.equal(kp[n_pages - 3, :, 100:105], more[0]) and torch.equal(vp[n_pages - 3, :, 100:105], more[0])
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_and_eviction_past_32_bits(cuda_device, dtype):
    """The same with scores: a step and an eviction in pages behind the border, which move nothing and touch no score elsewhere."""
    page, d, hkv, G, dt = 1024, 128, 4, 2, DT[dtype]
    n_pages = (1 << 31) // (page * d * hkv) + 8
    kp = torch.zeros(n_pages, hkv, page, d, dtype=dt, device="cuda")
    vp = torch.zeros_like(kp)
    pos, score = torch.zeros(n_pages, hkv, page, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, hkv, page, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(4)
    table = torch.tensor([[n_pages - 1, 1, n_pages - 4]], dtype=torch.int32, device="cuda")
    n, keep = 2 * page + 77, 900
    for i, p in enumerate(table[0].tolist()):
        kp[p], vp[p] = (torch.randn(hkv, page, d, generator=g, device="cuda").to(dt) for _ in range(2))
        pos[p] = torch.arange(i * page, (i + 1) * page, device="cuda", dtype=torch.int32)
    length = torch.full((1, hkv), n, dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(1, h, d, generator=g, device="cuda").to(dt) for h in (hkv * G, hkv, hkv))
    out = torch.empty_like(q)
    c = B.D2OPagedCache(kp, vp, table, length, n_q_heads=hkv * G, pos=pos, score=score)
    c.d2o_paged_decode_step(q, k, v, out)
    dense = lambda pool: pool[table[0].long()].transpose(0, 1).flatten(1, 2)[:, :n + 1]
    K, V = dense(kp).double(), dense(vp).double()
    assert torch.equal(K[:, n], k[0].double()) and torch.equal(V[:, n], v[0].double())
    p = torch.softmax(torch.einsum("hgd,hnd->hgn", q[0].double().view(hkv, G, d), K) / math.sqrt(d), -1)
    torch.testing.assert_close(out[0].double().view(hkv, G, d), p @ V, rtol=2.0 ** -8, atol=1e-5)
    torch.testing.assert_close(dense(score).double(), p.sum(1), rtol=1e-4, atol=1e-9)
    assert int((score != 0).sum()) == hkv * (n + 1)
    length += 1
    was_k, was_v, was_s, was_p = (dense(t).clone() for t in (kp, vp, score, pos))
    c.d2o_paged_evict(torch.full((1, hkv), keep, dtype=torch.int32, device="cuda"), torch.tensor([n + 1], dtype=torch.int32, device="cuda"), n_sink=2, window=50)
    rank = was_s.double() + ((was_p < 2) | (was_p >= n + 1 - 50)) * 1e9 - was_p.double() * 1e-18
    for h in range(hkv):
        stays = torch.zeros(n + 1, dtype=torch.bool, device="cuda")
        stays[rank[h].topk(keep).indices] = True
        to, frm = (~stays[:keep]).nonzero()[:, 0], stays[keep:].nonzero()[:, 0] + keep
        src = torch.arange(keep, device="cuda")
        src[to] = frm
        for pool, was in ((kp, was_k), (vp, was_v), (score, was_s), (pos, was_p)):
            assert torch.equal(dense(pool)[h, :keep], was[h, src]) and torch.equal(dense(pool)[h, keep:], was[h, keep:])
    c.check()


# ---------------------------------------------------------------------------------------------- many, at once, and with one scratch
def _batch(seed, b, hkv, G, d, dtype, page, held, scored=False):
    """A cache made on the GPU, lengths 0 .. held; returns it with its tensors and a function for the float64 output of one slice."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    per = held // page + 1
    n_pages = b * per + 1
    table = torch.randperm(n_pages, generator=g, device="cuda")[: b * per].view(b, per).to(torch.int32)
    kp, vp = (torch.randn(n_pages, hkv, page, d, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    length = torch.randint(0, held + 1, (b, hkv), generator=g, device="cuda", dtype=torch.int32)
    q, k, v = (torch.randn(b, h, d, generator=g, device="cuda").to(DT[dtype]) for h in (hkv * G, hkv, hkv))
    pos = torch.zeros(n_pages, hkv, page, dtype=torch.int32, device="cuda") if scored else None
    score = torch.zeros(n_pages, hkv, page, device="cuda") if scored else None
    c = B.D2OPagedCache(kp, vp, table, length, n_q_heads=hkv * G, pos=pos, score=score)

    def check(out, slices):
        for i, h in slices:
            n = int(length[i, h])
            rows = lambda pool: pool[table[i].long(), h].flatten(0, 1)[: n + 1].double()
            K, V, Q = rows(kp), rows(vp), q[i, h * G:(h + 1) * G].double()
            assert torch.equal(K[n], k[i, h].double()) and torch.equal(V[n], v[i, h].double())
            p = torch.softmax(Q @ K.T / math.sqrt(d), -1)
            w = 32 * 2.0 ** -24 * float((Q.abs() @ K.abs().T).max()) / math.sqrt(d) + 2.0 ** -20
            e, ref = (w + (2.0 ** -16 if dtype == "bf16" else 0)) * (p @ V.abs()), p @ V
            o = out[i, h * G:(h + 1) * G].double()
            assert bool((((ref - e).to(DT[dtype]).double() <= o) & (o <= (ref + e).to(DT[dtype]).double())).all()), (i, h, n)
    return c, q, k, v, torch.full_like(q, NAN), check


@pytest.mark.parametrize("b,hkv,G,d,dtype,held", [(8191, 8, 1, 64, "f16", 15), (8191, 8, 1, 64, "f32", 15), (600, 8, 2, 128, "bf16", 100), (40, 8, 4, 128, "bf16", 3000),
                                                  (40, 8, 8, 128, "f16", 900), (9, 2, 8, 64, "f32", 2500), (150, 1, 1, 128, "bf16", 700)])
def test_decode_many(cuda_device, b, hkv, G, d, dtype, held):
    """The most slices, more slices than SMs of lengths around the borders of the shares, every group size."""
    c, q, k, v, out, check = _batch(b + held, b, hkv, G, d, dtype, 16, held)
    c.d2o_paged_decode_step(q, k, v, out)
    assert bool(torch.isfinite(out.float()).all())
    g = torch.Generator().manual_seed(1)
    check(out, [(int(i), int(i) % hkv) for i in torch.randint(0, b, (60,), generator=g)] + [(0, 0), (b - 1, hkv - 1)])
    again = torch.empty_like(out)
    c.d2o_paged_decode_step(q, k, v, again)
    assert torch.equal(out, again)
    c.check()
    zero = c._scratch[0] - c.scratch.data_ptr()
    assert not c.scratch[zero:zero + B.PAGED_ZERO_BYTES].any()                 # as every call leaves them


@pytest.mark.parametrize("dtype,d,G", [("bf16", 128, 4), ("f16", 64, 1), ("bf16", 64, 8), ("f16", 128, 2)])
def test_decode_clusters_of_idle_warps(cuda_device, dtype, d, G):
    """Slices with a cluster each and a tile or two in all, so that most warps, and whole CTAs, have nothing to do and are at the shared barriers
    first: many launches in a row, nothing lost, the same bits."""
    c, q, k, v, out, check = _batch(d + G, 2, 4, G, d, dtype, 16, 40)
    check_all = [(i, h) for i in range(2) for h in range(4)]
    for n in (0, 1, 15, 16, 40):
        c.tensors[3].fill_(n)
        c.d2o_paged_decode_step(q, k, v, out)
        check(out, check_all)
        outs = torch.zeros(200, *q.shape, dtype=q.dtype, device="cuda")
        for x in outs:
            c.d2o_paged_decode_step(q, k, v, x)
        c.check()
        assert bool((outs == out).all())


def test_streams_at_once(cuda_device):
    """Steps on two caches, an eviction on a third and a prompt's attention, on four streams at the same time, many times over: the bits
    of the same calls one after another."""
    a = _batch(1, 20, 8, 4, 128, "bf16", 16, 1500)
    b = _batch(2, 3, 8, 1, 64, "f32", 32, 4000)
    Q, K, V = (torch.randn(2, h, 500, 128, device="cuda").half() for h in (8, 2, 2))
    want = []
    for c, q, k, v, out, _ in (a, b):
        c.d2o_paged_decode_step(q, k, v, out, window=700, n_sink=3)
        want.append(out.clone())
    o = torch.empty_like(Q)
    B.d2o_prompt_attention(Q, K, V, o, window=100, n_sink=2)
    want.append(o.clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(20):
        for t in (a[4], b[4], o):
            t.zero_()
        torch.cuda.synchronize()
        for st, x in zip(streams, (a, b)):
            with torch.cuda.stream(st):
                for _ in range(3):
                    x[0].d2o_paged_decode_step(x[1], x[2], x[3], x[4], window=700, n_sink=3)
        with torch.cuda.stream(streams[2]):
            for _ in range(3):
                B.d2o_prompt_attention(Q, K, V, o, window=100, n_sink=2)
        torch.cuda.synchronize()
        assert torch.equal(a[4], want[0]) and torch.equal(b[4], want[1]) and torch.equal(o, want[2])


def test_scores_and_evictions_on_streams_at_once(cuda_device):
    """Two caches with scores that take steps, one of them between evictions, a third that is evicted from, and a prompt's attention, on four streams
    at the same time, many times over: the bits of the same calls one after another."""
    a = _batch(11, 20, 8, 4, 128, "bf16", 16, 1500, True)
    b = _batch(12, 3, 8, 1, 64, "f32", 32, 4000, True)
    e = _batch(13, 5, 8, 2, 128, "f16", 16, 9000, True)
    Q, K, V = (torch.randn(2, h, 700, 128, device="cuda").half() for h in (8, 2, 2))
    o = torch.empty_like(Q)
    g = torch.Generator(device="cuda").manual_seed(1)
    for x in (a, b, e):
        pos, score = x[0].tensors[4:6]
        pos.copy_(torch.randint(0, 1 << 20, pos.shape, generator=g, device="cuda"))
        score.copy_(torch.rand(score.shape, generator=g, device="cuda"))
    pools = [[x[0].tensors[j] for j in (0, 1, 4, 5)] for x in (a, b, e)]
    kept = [[t.clone() for t in ts] for ts in pools]
    next_pos = {id(x): torch.full((x[0].shape[0],), 1 << 19, dtype=torch.int32, device="cuda") for x in (a, b, e)}
    budgets = {id(x): (x[0].tensors[3] // 3).contiguous() for x in (a, b, e)}

    def steps(x):
        for _ in range(3):
            x[0].d2o_paged_decode_step(x[1], x[2], x[3], x[4])

    def evict(x):
        x[0].d2o_paged_evict(budgets[id(x)], next_pos[id(x)], n_sink=100, window=50)

    def between():
        steps(a)
        evict(a)
        steps(a)
    jobs = [between, lambda: steps(b), lambda: evict(e), lambda: B.d2o_prompt_attention(Q, K, V, o, window=100, n_sink=2)]
    results = lambda: [t for ts in pools for t in ts] + [a[4], b[4], o]

    def restore():
        for ts, ks in zip(pools, kept):
            for t, k in zip(ts, ks):
                t.copy_(k)
        for t in (a[4], b[4], o):
            t.zero_()
        torch.cuda.synchronize()
    restore()
    for job in jobs:
        job()
        torch.cuda.synchronize()
    want = [t.clone() for t in results()]
    assert not torch.equal(want[2], kept[0][2]) and not torch.equal(want[10], kept[2][2])      # evictions moved rows
    streams = [torch.cuda.Stream() for _ in jobs]
    for turn in range(12):
        restore()
        for i in range(4):
            with torch.cuda.stream(streams[(i + turn) % 4]):
                jobs[(i + turn) % 4]()
        torch.cuda.synchronize()
        for t, w in zip(results(), want):
            assert np.array_equal(bits(t), bits(w))
    for x in (a, b, e):
        x[0].check()


def test_made_on_one_stream_used_on_another(cuda_device):
    """The scratch is cleared when the constructor returns, also behind work that is under way on its stream."""
    a = _batch(3, 20, 8, 4, 128, "bf16", 16, 1500)
    a[0].d2o_paged_decode_step(a[1], a[2], a[3], a[4])
    want, size = a[4].clone(), a[0].scratch.numel()
    k, v, table, length, _, _ = a[0].tensors
    x = torch.randn(8192, 8192, device="cuda")
    torch.full((size,), 255, dtype=torch.uint8, device="cuda")                 # what the next allocation of this size may find
    torch.cuda.synchronize()
    for _ in range(4):
        x @ x
    c = B.D2OPagedCache(k, v, table, length, n_q_heads=32)
    assert torch.cuda.current_stream().query()
    side, out = torch.cuda.Stream(), torch.zeros_like(want)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.d2o_paged_decode_step(a[1], a[2], a[3], out)
    c.check()                                                                  # waits for the side stream too
    assert torch.equal(out, want)


def test_one_scratch_for_several_caches(cuda_device):
    """Caches of other shapes in turn on one scratch, as large as the largest asks for."""
    caches = [_batch(i, b, hkv, G, d, dt, 16, held, True) for i, (b, hkv, G, d, dt, held) in enumerate(
        [(30, 8, 4, 128, "bf16", 900), (1, 1, 1, 64, "f32", 20000), (700, 2, 2, 64, "f16", 40)])]
    big = max(caches, key=lambda x: x[0]._scratch[1])[0]
    for _ in range(2):
        for c, q, k, v, out, check in caches:
            c._scratch = big._scratch
            c.d2o_paged_decode_step(q, k, v, out)
            b, hkv = c.tensors[3].shape
            check(out, [(i, i % hkv) for i in range(0, b, max(1, b // 8))])
            c.d2o_paged_evict((c.tensors[3] + 1).contiguous(), torch.full((b,), 30000, dtype=torch.int32, device="cuda"))     # nothing to do
            c.check()


def test_steps_and_evictions_of_several_caches_on_one_scratch(cuda_device):
    """Steps with scores and evictions that move rows, of caches of other shapes in turn, through one scratch (the logits of one lie where the moves of the
    other do): every pool against the plain statements."""
    shapes = [(2, 4, 2, 64, "bf16", 16, [90, 61]), (1, 8, 1, 128, "f16", 32, [200]), (3, 2, 2, 64, "f32", 16, [40, 75, 3])]
    caches = [Paged(i, b, hq, hkv, d, dt, page, max(held) // page + 2, held) for i, (b, hq, hkv, d, dt, page, held) in enumerate(shapes)]
    big = max((c.cache for c in caches), key=lambda c: c._scratch[1])
    for c in caches:
        c.cache._scratch = big._scratch
    for turn in range(3):
        for c in caches:
            q, k, v = c.randn(c.b, c.hq, c.d), c.randn(c.b, c.hkv, c.d), c.randn(c.b, c.hkv, c.d)
            out = torch.full((c.b, c.hq, c.d), 3.0, dtype=c.dt, device="cuda")
            c.cache.d2o_paged_decode_step(q.cuda(), k.cuda(), v.cuda(), out)
            c.step(q, k, v, out, None, 0, 0)
            c.same()
            c.len += 1
            c.dlen.copy_(c.len)
        for c in caches:
            budgets, next_pos = (c.len * 2 // 3).to(torch.int32), c.len.amax(1).to(torch.int32)
            c.cache.d2o_paged_evict(budgets.cuda(), next_pos.cuda(), n_sink=1, window=5)
            c.evict(budgets, next_pos, 1, 5)
            c.same()
            c.len = torch.minimum(c.len, budgets)
            c.dlen.copy_(c.len)
            c.cache.check()


# ---------------------------------------------------------------------------------------------- evict
@pytest.mark.parametrize("b,hq,hkv,d,dtype,page,held,budget,window,sinks", [
    (1, 1, 1, 64, "f32", 16, [1], [0], 0, 0), (1, 1, 1, 64, "f32", 16, [2], [1], 0, 0), (1, 2, 2, 128, "bf16", 16, [40], [39], 4, 1),
    (2, 4, 2, 128, "f16", 16, [100, 33], [25, 32], 8, 2), (3, 4, 1, 64, "bf16", 32, [200, 5, 64], [64, 10, 64], 16, 4),
    (2, 8, 8, 128, "f32", 64, [150, 151], [149, 3], 2, 1), (1, 4, 2, 64, "f16", 16, [700], [350], 0, 0), (2, 2, 2, 64, "bf16", 16, [-1, 90], [4, 80], 79, 1),
    (1, 1, 1, 64, "f16", 128, [2100], [1], 0, 0), (1, 1, 1, 64, "bf16", 16, [600], [300], 1000, 0)])
@pytest.mark.parametrize("kind", ["spread", "ties", "zeros", "special", "shuffled"])
def test_evict(cuda_device, b, hq, hkv, d, dtype, page, held, budget, window, sinks, kind):
    c = Paged(sum(held) + 1, b, hq, hkv, d, dtype, page, max(1, (max(held) + page - 1) // page), held)
    s = c.score
    if kind == "ties":
        s.copy_(torch.where(s == s, (s * 4).floor(), s))
    elif kind == "zeros":
        s.copy_(torch.where(s == s, torch.where(s < 0.5, 0.0, -0.0), s))
    elif kind == "special":
        x = torch.rand(s.shape, generator=c.g)
        s.copy_(torch.where(x < 0.1, NAN, torch.where(x < 0.2, -NAN, torch.where(x < 0.3, math.inf, torch.where(x < 0.5, -math.inf, torch.where(x < 0.6, -s, s))))))
    elif kind == "shuffled":                                                   # positions in another order, with gaps
        s.copy_(torch.where(s == s, (s * 8).floor(), s))
        for i in range(b):
            for h in range(hkv):
                p = torch.randperm(2 * max(1, held[i]), generator=c.g)
                for r in range(max(0, held[i])):
                    pg, at = c.at(i, r)
                    c.pos[pg, h, at] = int(p[r])
    c.upload()
    next_pos = torch.tensor([max(0, x) * (2 if kind == "shuffled" else 1) for x in held], dtype=torch.int32)
    budgets = torch.tensor(budget, dtype=torch.int32)[:, None].expand(b, hkv).contiguous()
    if hkv > 1:                                                                # heads with sizes of their own
        budgets[:, 1] = (budgets[:, 1] - 1).clamp(min=0)
    c.cache.d2o_paged_evict(budgets.cuda(), next_pos.cuda(), n_sink=sinks, window=window)
    c.evict(budgets, next_pos, sinks, window)
    c.same()
    c.cache.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 128), ("f16", 64)])
@pytest.mark.parametrize("held,budget", [([1, 0], [0, 0]), ([5, 300], [3, 41]), ([17, 16], [16, 15]), ([2, 40], [1, 39]), ([600, 1500], [1, 1499])])
def test_evict_few_rows_in_a_large_table(cuda_device, dtype, d, held, budget):
    """Tables with room for 33600 rows: clusters of sixteen, most of whose CTAs have no rows."""
    c = Paged(sum(held) + d, 2, 4, 2, d, dtype, 16, 2100, held)
    c.score.copy_(torch.where(c.score == c.score, (c.score * 6).floor(), c.score))
    c.table[:, (max(held) + 15) // 16:] = -1
    c.upload()
    budgets = torch.tensor(budget, dtype=torch.int32)[:, None].expand(2, 2).contiguous()
    next_pos = torch.tensor(held, dtype=torch.int32)
    c.cache.d2o_paged_evict(budgets.cuda(), next_pos.cuda(), n_sink=1, window=9)
    c.evict(budgets, next_pos, 1, 9)
    c.same()
    c.cache.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,max_pages", [(2, 4), (2, 4000), (700, 4)])
def test_no_sequences(cuda_device, dtype, b, max_pages):
    """A batch of padding alone: nothing is read or written."""
    c = Paged(3, b, 4, 2, 64, dtype, 16, max_pages, [-1] * b)
    out = torch.full((b, 4, 64), 3.0, dtype=c.dt, device="cuda")
    x = lambda *s: torch.zeros(*s, dtype=c.dt, device="cuda")
    for _ in range(2):
        c.cache.d2o_paged_decode_step(x(b, 4, 64), x(b, 2, 64), x(b, 2, 64), out)
        c.cache.d2o_paged_append(x(b, 2, 5, 64), x(b, 2, 5, 64))
        c.cache.d2o_paged_evict(torch.zeros(b, 2, dtype=torch.int32, device="cuda"), torch.zeros(b, dtype=torch.int32, device="cuda"))
    assert bool((out == 3).all())
    c.same()
    c.cache.check()


@pytest.mark.parametrize("held,budget", [(40, 9), (90, 25), (700, 15), (2000, 1100)])
def test_evict_positions_below_zero(cuda_device, held, budget):
    """Positions around zero, as a padded batch may count them: all below n_sink are protected, and the budget is spent on the earliest of them; and ties
    of ordinary rows on both sides of zero."""
    c = Paged(held, 2, 4, 2, 64, "bf16", 16, (held + 15) // 16, [held, held - 1])
    c.pos.copy_(torch.where(c.pos == -7, c.pos, c.pos - 17))
    c.score.copy_(torch.where(c.score == c.score, (c.score * 2).floor(), c.score))
    c.upload()
    budgets = torch.tensor([[budget, budget + 1], [budget - 1, 7]], dtype=torch.int32)
    next_pos = torch.tensor([held - 17, held - 18], dtype=torch.int32)
    c.cache.d2o_paged_evict(budgets.cuda(), next_pos.cuda(), n_sink=5, window=3)
    c.evict(budgets, next_pos, 5, 3)
    c.same()
    c.cache.check()


@pytest.mark.parametrize("n,budget,b,hkv", [(30000, 6000, 1, 8), (30001, 29990, 1, 1), (20000, 3000, 40, 8)])
def test_evict_long(cuda_device, n, budget, b, hkv):
    """More rows than shared memory keeps keys of, ties at the border; checked on the GPU."""
    page, d, dt = 64, 64, torch.float16
    g = torch.Generator(device="cuda").manual_seed(n)
    per = (n + page - 1) // page
    table = torch.randperm(per * b + 1, generator=g, device="cuda")[: per * b].view(b, per).to(torch.int32)
    shape = (per * b + 1, hkv, page)
    pos = torch.zeros(shape, dtype=torch.int32, device="cuda")
    slot = torch.arange(per * page, device="cuda").expand(b, hkv, -1)
    flip = (n - 1 - slot).clamp(min=0).to(torch.int32)                         # positions against the order of the rows
    pos[table.long()] = flip.view(b, hkv, per, page).transpose(1, 2)
    score = (torch.rand(shape, generator=g, device="cuda") * 50).floor()
    # a row's K and V name the row
    kp = (torch.rand(*shape, 1, generator=g, device="cuda")).to(dt).expand(*shape, d).contiguous()
    vp = (-kp).contiguous()
    dense = lambda pool: pool[table.long()].transpose(1, 2).flatten(2, 3)
    key = dense(score)[..., :n].double() * (1 << 20) - flip[..., :n].double()
    key[..., n - 3:] += 1e15                                                   # positions 0 .. 2: sinks
    want = torch.zeros(b, hkv, n, dtype=torch.bool, device="cuda").scatter_(-1, key.topk(budget).indices, True)
    want_pos = dense(pos)[..., :n].clone()
    for i in range(b):
        for h in range(hkv):
            to, frm = (~want[i, h, :budget]).nonzero()[:, 0], want[i, h, budget:].nonzero()[:, 0] + budget
            want_pos[i, h, to] = want_pos[i, h, frm]
    was = {p: dense(p_).clone() for p, p_ in (("k", kp), ("score", score))}
    c = B.D2OPagedCache(kp, vp, table, torch.full((b, hkv), n, dtype=torch.int32, device="cuda"), n_q_heads=hkv, pos=pos, score=score)
    c.d2o_paged_evict(torch.full((b, hkv), budget, dtype=torch.int32, device="cuda"), torch.full((b,), n, dtype=torch.int32, device="cuda"), n_sink=3)
    got = dense(pos)[..., :n]
    assert torch.equal(got, want_pos)
    src = (n - 1 - got).long()                                                 # the row that each row's contents came from
    assert torch.equal(dense(score)[..., :n], was["score"].gather(-1, src))
    assert torch.equal(dense(kp)[..., :n, 3], was["k"][..., 3].gather(-1, src)) and torch.equal(dense(vp)[..., :n, :], -dense(kp)[..., :n, :])
    c.check()


# ---------------------------------------------------------------------------------------------- anomalies
@pytest.mark.parametrize("n", [1500, 30000])
def test_evict_same_pages_in_two_tables(cuda_device, n):
    """Against the documentation: what the pools hold afterwards is undefined, what lies around them stays, and later calls are right."""
    page, d, hkv = 16, 64, 2
    per = (n + page - 1) // page
    g = torch.Generator(device="cuda").manual_seed(n)
    guard = 4 * hkv * page * d
    pools = [torch.full((2 * guard + (per + 1) * hkv * page * w,), 5, dtype=dt, device="cuda") for w, dt in ((d, torch.float16), (d, torch.float16), (1, torch.int32), (1, torch.float32))]
    inner = [x[guard:-guard] for x in pools]
    kp, vp = (x.view(per + 1, hkv, page, d) for x in inner[:2])
    pos, score = (x.view(per + 1, hkv, page) for x in inner[2:])
    pos.copy_(torch.randint(0, 1 << 20, pos.shape, generator=g, device="cuda"))
    table = torch.randperm(per + 1, generator=g, device="cuda")[:per].to(torch.int32).expand(4, per).contiguous()
    length = torch.full((4, hkv), n, dtype=torch.int32, device="cuda")
    c = B.D2OPagedCache(kp, vp, table, length, n_q_heads=hkv, pos=pos, score=score)
    c.scratch[B.PAGED_ZERO_BYTES + 256:].fill_(0x7F)                           # entries that no call wrote name rows far outside
    budgets = torch.tensor([n // 5, n // 2, n // 3, n - 7], dtype=torch.int32, device="cuda")[:, None].expand(4, hkv).contiguous()
    for _ in range(3):
        c.d2o_paged_evict(budgets, torch.full((4,), 1 << 20, dtype=torch.int32, device="cuda"))
    c.check()
    for x in pools:
        assert bool((x[:guard] == 5).all()) and bool((x[-guard:] == 5).all())
    test_evict_long(cuda_device, 20000, 3000, 1, 8)


def test_bad_tables(cuda_device):
    """Page numbers out of range and tables that are too short: reported, nothing read or written through them; other sequences go on."""
    def fresh():
        c = Paged(4, 3, 4, 2, 64, "bf16", 16, 3, [40, 40, 47])
        c.table[1, 1] = 99
        return c
    up = lambda t: t.cuda()
    c = fresh()
    c.upload()
    q, k, v = c.randn(3, 4, 64), c.randn(3, 2, 64), c.randn(3, 2, 64)
    out = torch.full((3, 4, 64), 3.0, dtype=c.dt, device="cuda")
    c.cache.d2o_paged_decode_step(up(q), up(k), up(v), out)
    assert bool(out[1].isnan().all()) and bool(torch.isfinite(out[0].float()).all()) and bool(torch.isfinite(out[2].float()).all())
    with pytest.raises(B.D2OError) as e:
        c.cache.check()
    assert e.value.status == 4
    c.cache.check()                                                            # the word has been taken
    c = fresh()
    c.table[1, 1] = -1
    c.len[2] = 48                                                              # row 48 has no page
    c.upload()
    c.cache.d2o_paged_decode_step(up(q), up(k), up(v), out)
    assert bool(out[1].isnan().all()) and bool(out[2].isnan().all()) and bool(torch.isfinite(out[0].float()).all())
    with pytest.raises(B.D2OError):
        c.cache.check()
    # append: what has a page is written
    c = fresh()
    c.len[1] = 10
    c.upload()
    K, V = c.randn(3, 2, 9, 64), c.randn(3, 2, 9, 64)
    c.cache.d2o_paged_append(up(K), up(V))
    for h in range(2):
        got = c.dk.cpu()
        assert torch.equal(got[int(c.table[1, 0]), h, 10:], K[1, h, :6]) and torch.equal(got[int(c.table[2, 2]), h, 15], K[2, h, 0])
        assert torch.equal(got[int(c.table[0, 2]), h, 8:], K[0, h, :8])
    was, now = (c.k == c.k).all(-1), (c.dk.cpu() == c.dk.cpu()).all(-1)
    assert int((now & ~was).sum()) == 2 * 1 + 2 * 8 and bool((was <= now).all())          # sequence 1 held 40 rows in the fixture
    with pytest.raises(B.D2OError):
        c.cache.check()
    # evict: the slice stays as it was
    c = fresh()
    c.upload()
    c.len[2] = 49
    c.dlen.copy_(c.len)
    budgets = torch.full((3, 2), 20, dtype=torch.int32)
    c.cache.d2o_paged_evict(up(budgets), torch.full((3,), 40, dtype=torch.int32, device="cuda"))
    keep = c.len.clone()
    c.len[1:] = -1
    c.evict(budgets, torch.full((3,), 40), 0, 0)
    c.len.copy_(keep)
    c.same()
    with pytest.raises(B.D2OError):
        c.cache.check()
    c.upload()
    c.cache.d2o_paged_evict(torch.full((3, 2), -1, dtype=torch.int32, device="cuda"), torch.full((3,), 40, dtype=torch.int32, device="cuda"))
    with pytest.raises(B.D2OError):
        c.cache.check()


# ---------------------------------------------------------------------------------------------- together
def test_serving_run(cuda_device):
    """Prompt attention -> column sums -> pages -> decode steps and evictions in turn, from a captured graph and without one: the same
    bits; every step against the plain statements."""
    b, hq, hkv, d, n, page, budget = 2, 8, 2, 128, 150, 16, 96
    lens = torch.tensor([150, 121], dtype=torch.int32)
    g = torch.Generator(device="cuda").manual_seed(8)
    Q, K, V = (torch.randn(b, h, n, d, generator=g, device="cuda").to(torch.bfloat16) for h in (hq, hkv, hkv))
    lse, out_p = torch.zeros(b, hq, n, device="cuda"), torch.zeros_like(Q)
    B.d2o_prompt_attention(Q, K, V, out_p, lse=lse, lens=lens.cuda())
    ctx = B.D2OContext(B.make_config(n_layers=1, batch=b, n_q_heads=hq, n_kv_heads=hkv, d_head=d, dtype="bf16", prompt_len=n,
                                     max_new_tokens=1, rho=0.5))
    ctx.d2o_set_prompt_lens(lens)
    ctx.d2o_layer_stats(0, Q, K, lse)
    colsum = ctx.colsum(0).clone()
    runs = []
    for graph in (False, True):
        c = Paged(5, b, hq, hkv, d, "bf16", page, 12, [0, 0])
        c.cache.d2o_paged_append(K, V, lens=lens.cuda(), colsum=colsum)
        c.append(K.cpu(), V.cpu(), lens, None, colsum.cpu())
        c.same()
        c.len += lens[:, None]
        c.dlen.copy_(c.len)
        seen = lens.clone()
        dseen, budgets = seen.cuda(), torch.full((b, hkv), budget, dtype=torch.int32, device="cuda")
        q, k, v = (torch.zeros(b, h, d, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
        out, g0, outs = torch.zeros_like(q), None, []

        def token():
            c.cache.d2o_paged_decode_step(q, k, v, out, positions=dseen)
            c.dlen.add_(1)
            dseen.add_(1)
            c.cache.d2o_paged_evict(budgets, dseen, n_sink=1, window=24)
            c.dlen.copy_(torch.minimum(c.dlen, budgets))
        for step in range(5):
            for x, h in ((q, hq), (k, hkv), (v, hkv)):
                x.copy_(c.randn(b, h, d))
            if graph and step == 0:
                keep = [t.clone() for t in (c.dk, c.dv, c.dpos, c.dscore, c.dlen, dseen)]
                s = torch.cuda.Stream()
                s.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(s):
                    token()                                                    # once outside of the capture
                torch.cuda.current_stream().wait_stream(s)
                for t, was in zip((c.dk, c.dv, c.dpos, c.dscore, c.dlen, dseen), keep):
                    t.copy_(was)
                g0 = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g0):
                    token()
            g0.replay() if graph else token()
            torch.cuda.synchronize()
            outs.append(out.clone())
            if not graph:
                dk = [t.clone() for t in (c.dk, c.dv, c.dpos, c.dscore)]
                # the scores moved with the rows: compare the step by itself on a second cache
                two = Paged(5, b, hq, hkv, d, "bf16", page, 12, [0, 0])
                two.k, two.v, two.pos, two.score, two.len, two.table = c.k, c.v, c.pos, c.score, c.len, c.table
                two.upload()
                two.cache.d2o_paged_decode_step(q, k, v, out, positions=seen.cuda())
                two.step(q.cpu(), k.cpu(), v.cpu(), out, seen, 0, 0)
                two.same()
                c.len += 1
                seen = seen + 1
                c.evict(budgets.cpu(), seen, 1, 24)
                c.len.clamp_(max=budget)
                assert all(np.array_equal(bits(x), bits(y)) for x, y in zip(dk, (c.k, c.v, c.pos, c.score)))
                c.same()
                assert torch.equal(dseen.cpu(), seen)
        c.cache.check()
        runs.append((outs, [bits(t) for t in (c.dk, c.dv, c.dpos, c.dscore)]))
    assert all(torch.equal(x, y) for x, y in zip(runs[0][0], runs[1][0]))
    assert all(np.array_equal(x, y) for x, y in zip(runs[0][1], runs[1][1]))
    ctx.close()
