"""Attention of runs of rows (socket_attend_rows) and the masses of keys (socket_key_mass) against plain 64-bit
arithmetic on the CPU.

Tolerances, derived from the arithmetic (u = 2^-24, half a step of fp32):
  logits   a dot product of d terms in fp32 is off by at most (d + 1) u sum |q_c k_c|; capping, bias and the change to
           units of log 2 add a few u of the logit's size, counted as 16 u (|s| + slope |i - j|).  Call the largest of
           these over a row's keys e: weights, and sums of weights, are off by at most 2 e + 2 e^2 of themselves.
  weights  exp2 and the running rescales: 8 u each; sums over n keys in fp32: n u.
  out      A = sum p |v|: off by A (4 e + (2 n + 32) u); bf16 outputs from weights rounded to bf16 add 2^-8 A for
           those, and 2^-8 |y| for their own rounding.
  lse      off by 2 e + (n + 32) u + 8 u |lse|;  masses by m (4 e + (n_queries + 64) u + 8 u max |lse|).
"""
import math

import numpy as np
import pytest
import torch

from paper_2602_06283_amd import binding as sk

U = 2.0 ** -24
HALF_BF16 = 2.0 ** -8


def bf16(x):
    return x.to(torch.bfloat16).double()


class Run:
    """A cache with runs appended, on the CPU in 64 bits (values exact in the cache's type) and on the device."""

    def __init__(self, seed, begins, counts, G=4, Hkv=2, d=128, f32=False, page=0, scale=None, softcap=0.0, window=0,
                 bias=False, prefix=None, docs=None, spare=0, logit_gain=1.0, max_rows=None):
        g = torch.Generator().manual_seed(seed)
        self.begins, self.counts, self.G, self.Hkv, self.Hq, self.d, self.f32, self.page = begins, counts, G, Hkv, G * Hkv, d, f32, page
        self.B = len(begins)
        unit = page or 16
        self.n = (max(b + c for b, c in zip(begins, counts)) + spare + unit - 1) // unit * unit
        self.R = max_rows if max_rows is not None else max(1, max(counts))
        self.scale = 1.0 / math.sqrt(d) if scale is None else scale
        self.softcap, self.window = softcap, window
        keep = (lambda x: x.float().double()) if f32 else bf16
        self.K = keep(torch.randn(self.B, Hkv, self.n, d, generator=g) * torch.exp(0.5 * torch.randn(Hkv, 1, d, generator=g)))
        self.V = keep(torch.randn(self.B, Hkv, self.n, d, generator=g))
        self.q = keep(logit_gain * torch.randn(self.B, self.R, self.Hq, d, generator=g))
        self.slopes = (2.0 ** (-8.0 * (torch.arange(self.Hq) + 1) / self.Hq)).float().double() if bias else None
        self.prefix = None if prefix is None else torch.tensor(prefix, dtype=torch.int32)
        self.docs = None
        if docs is not None:            # cut points -> first token of each token's document
            cuts = np.array([0] + list(docs))
            at = cuts[np.searchsorted(cuts, np.arange(self.n), side="right") - 1]
            self.docs = torch.from_numpy(np.tile(at, (self.B, 1)).astype(np.int32))
        self.table = None
        if page:
            blocks = self.n // page
            self.table = torch.randperm(self.B * blocks + 3, generator=g)[: self.B * blocks].view(self.B, blocks).to(torch.int32)
            self.num_blocks = self.B * blocks + 3

    # -- the definition
    def seen(self, b):
        """[rows, n] which keys each row of sequence b sees."""
        begin, count = self.begins[b], self.counts[b]
        i = torch.arange(begin, begin + count)[:, None]
        j = torch.arange(self.n)[None]
        lo, hi = torch.zeros_like(i), i.clone()
        if self.window:
            lo = torch.maximum(lo, i - self.window + 1)
        if self.docs is not None:
            lo = torch.maximum(lo, self.docs[b][begin:begin + count, None].long())
        if self.prefix is not None:
            hi = torch.maximum(hi, (self.prefix[b] - 1).long().expand_as(hi))
        hi = hi.clamp(max=begin + count - 1)
        ok = (j >= lo) & (j <= hi)
        if self.table is not None:
            gone = (self.table[b] < 0) | (self.table[b] >= self.num_blocks)
            ok &= ~gone.repeat_interleave(self.page)[None, : self.n]
        return ok

    def logits(self, b, hq):
        """Logits of the rows of (b, hq), -inf where not seen, and how far a kernel's may be off."""
        begin, count = self.begins[b], self.counts[b]
        q, K = self.q[b, :count, hq], self.K[b, hq // self.G]
        ok = self.seen(b)
        Kz = torch.where(ok.any(0)[:, None], K, torch.zeros_like(K)).nan_to_num(0.0, 0.0, 0.0)
        s = q @ Kz.T * self.scale
        off = (self.d + 1) * U * (q.abs() @ Kz.abs().T) * abs(self.scale)
        if self.softcap:
            s = self.softcap * torch.tanh(s / self.softcap)
        size = s.abs()
        if self.slopes is not None:
            bias = self.slopes[hq] * (torch.arange(begin, begin + count)[:, None] - torch.arange(self.n)).abs()
            s, size = s - bias, size + bias
        off = torch.where(ok, off + 16 * U * size, torch.zeros_like(off)).amax(-1)
        return s.masked_fill(~ok, -math.inf), off

    def attention(self):
        """out, lse [B, R, ..] and their tolerances for an fp32 output and for a bf16 one."""
        out = torch.zeros(self.q.shape, dtype=torch.float64)
        lse = torch.zeros(self.q.shape[:3], dtype=torch.float64)
        t32, t16, tl = torch.zeros_like(out), torch.zeros_like(out), torch.zeros_like(lse)
        for b in range(self.B):
            c = self.counts[b]
            for hq in range(self.Hq if c else 0):
                s, e = self.logits(b, hq)
                used = torch.isfinite(s).any(0)
                V = torch.where(used[:, None], self.V[b, hq // self.G], torch.zeros_like(self.V[b, hq // self.G]))
                lse[b, :c, hq] = torch.logsumexp(s, -1)
                p = torch.softmax(s, -1).nan_to_num(0.0)
                # (a row that does not see a key does not touch its value, also where another row does)
                bad = ~torch.isfinite(V).all(-1)
                y = p[:, ~bad] @ V[~bad]
                for j in torch.nonzero(bad).flatten().tolist():
                    rows = torch.isfinite(s[:, j])
                    y[rows] += p[rows, j, None] * V[j]
                A = p @ V.abs().nan_to_num(0.0, 0.0, 0.0)
                n = self.n
                out[b, :c, hq] = y
                t32[b, :c, hq] = A * (4 * e + (2 * n + 32) * U)[:, None]
                t16[b, :c, hq] = t32[b, :c, hq] + HALF_BF16 * A + HALF_BF16 * y.abs().nan_to_num(0.0, 0.0, 0.0)
                tl[b, :c, hq] = 2 * e + (n + 32) * U + 8 * U * lse[b, :c, hq].abs().nan_to_num(0.0, 0.0, 0.0)
        return out, lse, t32, t16, tl

    def masses(self, before, decay, last, lse):
        m = before.clone()
        tol = torch.zeros_like(m)
        for b in range(self.B):
            begin, c = self.begins[b], self.counts[b]
            if c == 0:
                continue
            first = max(0, c - last) if last else 0
            m[b, :, :begin] = m[b, :, :begin] * decay if decay else 0.0
            m[b, :, begin:begin + c] = 0.0
            tol[b, :, :begin] = 2 * U * m[b, :, :begin].abs()
            for hq in range(self.Hq):
                s, e = self.logits(b, hq)
                L = lse[b, :c, hq, None].double()
                w = torch.exp(s - torch.where(torch.isfinite(L), L, torch.zeros_like(L)))
                w = torch.where(torch.isfinite(L), w, torch.zeros_like(w))[first:]
                m[b, hq // self.G] += w.sum(0)
                far = 8 * U * L.abs().nan_to_num(0.0, 0.0, 0.0)[first:]
                tol[b, hq // self.G] += (w * (4 * e[first:, None] + (c * self.G + 64) * U + far)).sum(0)
        return m, tol

    # -- on the device
    def device(self, max_batch=None, max_k=16):
        dt = torch.float32 if self.f32 else torch.bfloat16
        self.dq, K, V = self.q.to(dt).cuda(), self.K.to(dt), self.V.to(dt)
        self.dtable = None
        if self.page:
            blocks = self.n // self.page
            pools = []
            for x in (K, V):
                pool = torch.full((self.num_blocks, self.Hkv, self.page, self.d), math.nan, dtype=dt)
                x = x.view(self.B, self.Hkv, blocks, self.page, self.d).transpose(1, 2)
                for b in range(self.B):
                    for s in range(blocks):
                        if 0 <= int(self.table[b, s]) < self.num_blocks:
                            pool[int(self.table[b, s])] = x[b, s]
                pools.append(pool)
            K, V = pools
            self.dtable = self.table.cuda()
        self.dK, self.dV = K.cuda(), V.cuda()
        self.dbegin, self.dcount = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (self.begins, self.counts))
        self.ctx = sk.Context(sk.make_params(self.d, self.Hq, self.Hkv, 16, 4, sk.F32 if self.f32 else sk.BF16,
                                             max_batch or self.B, self.n, min(max_k, self.n), self.page,
                                             self.n // self.page if self.page else 0, self.num_blocks if self.page else 0))
        self.mods = dict(softcap=self.softcap, window=self.window,
                         slopes=None if self.slopes is None else self.slopes.float().cuda(),
                         prefix_len=None if self.prefix is None else self.prefix.cuda(),
                         doc_begin=None if self.docs is None else self.docs.cuda(), block_table=self.dtable)
        return self

    def attend(self, out_f32=True, with_lse=True, stream=None):
        out = torch.full(self.dq.shape, 7.0, dtype=torch.float32 if out_f32 else torch.bfloat16, device="cuda")
        lse = torch.full(self.dq.shape[:3], 7.0, device="cuda") if with_lse else None
        torch.cuda.synchronize()
        self.ctx.attend_rows(self.dq, self.dK, self.dV, self.dbegin, self.dcount, self.B, self.R, self.scale, out, lse=lse,
                             stream=stream, **self.mods)
        return out, lse

    def check(self, out, lse=None, want=None):
        w, wl, t32, t16, tl = want or self.attention()
        tol = t32 if out.dtype == torch.float32 else t16
        got = out.cpu().double()
        for b in range(self.B):
            c = self.counts[b]
            x, y = got[b, :c], w[b, :c]
            assert torch.equal(torch.isnan(x), torch.isnan(y)), b
            fine = torch.isfinite(y)
            assert torch.equal(x[~fine & ~torch.isnan(y)], y[~fine & ~torch.isnan(y)])
            worst = ((x - y).abs() - tol[b, :c])[fine]
            assert worst.numel() == 0 or float(worst.max()) <= 0, (b, float(worst.max()))
            assert bool((got[b, c:] == 7.0).all()), "rows behind the run were written"
            if lse is not None:
                x, y = lse[b, :c].cpu().double(), wl[b, :c]
                assert torch.equal(torch.isinf(x), torch.isinf(y)) and not bool(torch.isnan(x).any() ^ torch.isnan(y).any())
                fine = torch.isfinite(y)
                worst = ((x - y).abs() - tl[b, :c])[fine]
                assert worst.numel() == 0 or float(worst.max()) <= 0, (b, float(worst.max()))
                assert bool((lse[b, c:].cpu() == 7.0).all())


SHAPES = [
    # begins, counts: one token, a few, ragged, runs of nothing, past tile borders
    dict(begins=[0], counts=[1]),
    dict(begins=[700], counts=[1]),
    dict(begins=[0, 63, 64, 501], counts=[1, 1, 1, 1]),
    dict(begins=[300, 0], counts=[5, 3]),
    dict(begins=[0], counts=[200]),
    dict(begins=[37, 130, 0], counts=[129, 0, 65]),
    dict(begins=[511], counts=[257]),
]
MODS = [
    dict(),
    dict(softcap=3.0, logit_gain=3.0),
    dict(softcap=50.0, bias=True),
    dict(window=33, bias=True),
    dict(prefix=[90] * 4, docs=[40, 170, 171, 400]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("mods", range(len(MODS)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("f32", [False, True])
def test_attention_of_runs(f32, shape, mods):
    m = dict(MODS[mods])
    if "prefix" in m:
        m["prefix"] = m["prefix"][: len(SHAPES[shape]["begins"])]
    run = Run(100 * shape + mods, f32=f32, page=[0, 16, 48][(shape + mods) % 3], **SHAPES[shape], **m).device()
    want = run.attention()
    run.check(*run.attend(True), want=want)
    run.check(*run.attend(False, with_lse=bool(mods % 2)), want=want)


@pytest.mark.gpu
@pytest.mark.parametrize("G,Hkv", [(1, 1), (1, 3), (2, 2), (4, 8), (8, 1)])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("f32", [False, True])
def test_heads_and_widths(f32, d, G, Hkv):
    run = Run(7 * d + G, [250, 3], [37, 70], G=G, Hkv=Hkv, d=d, f32=f32, page=16 if G == 2 else 0, softcap=20.0 if G == 4 else 0.0).device()
    want = run.attention()
    run.check(*run.attend(True), want=want)
    run.check(*run.attend(False), want=want)


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.0])
def test_any_scale(scale):
    for more in (dict(), dict(softcap=10.0, bias=True)):
        run = Run(5, [90, 0], [20, 33], scale=scale, **more).device()
        run.check(*run.attend(True))


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 2, 40])
@pytest.mark.parametrize("f32", [False, True])
def test_long_caches_are_split_and_joined(f32, rows):
    run = Run(11 + rows, [9001, 4444, 70], [rows, 1, rows], Hkv=1, G=2, d=64, f32=f32, page=16, softcap=30.0).device()
    run.check(*run.attend(True))


@pytest.mark.gpu
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rows", [1, 90])
def test_what_a_row_does_not_see_never_counts(f32, rows):
    """Infinities and NaN behind the sequence, in later rows, outside the window, in other documents and in absent
    blocks leave the result as the definition has it."""
    run = Run(21, [200, 96], [rows, rows], f32=f32, page=16, window=60, docs=[230], spare=40)
    for b in range(2):
        end = run.begins[b] + rows
        run.K[b, :, end:] = math.nan
        run.V[b, :, end:] = math.inf
        run.K[b, :, :30] = math.inf                      # outside every window
        run.V[b, :, :30] = math.nan
    if rows > 1:
        run.V[0, 0, 226, 5] = math.inf                   # the end of the first document: its own rows see it
        run.V[0, 1, 290 - 3] = -math.inf                 # seen by the last three rows alone
    run.table[1, 5] = -1                                 # tokens 80 .. 95 are not there
    run.table[0, 9] = run.num_blocks
    run.device()
    run.check(*run.attend(True))
    run.check(*run.attend(False))


@pytest.mark.gpu
def test_rows_that_see_nothing():
    run = Run(31, [50], [70], docs=[20])
    run.docs[0, 60:75] = 5000                            # documents that begin behind their tokens
    run.docs[0, 119] = 2 ** 31 - 1
    run.device()
    out, lse = run.attend(True)
    run.check(out, lse)
    assert bool((out[0, 10:25] == 0).all()) and bool(torch.isinf(lse[0, 10:25]).all())
    one = Run(32, [50], [1], docs=[])
    one.docs[0, 50] = 51
    one.device()
    out, lse = one.attend(False)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.gpu
def test_all_scores_minus_infinity_give_zeros():
    run = Run(33, [5], [2], Hkv=1, G=1, f32=True, scale=1.0)
    run.K[:] = -math.inf
    run.q[:] = 1.0
    run.device()
    out, lse = run.attend(True)
    assert bool((out[0, :2] == 0).all()) and bool((lse[0, :2] == -math.inf).all())


@pytest.mark.gpu
def test_runs_that_leave_the_cache_are_cut():
    run = Run(41, [10, 10, 10], [6, 6, 6], max_rows=6).device()
    run.dbegin.copy_(torch.tensor([run.n - 2, -1, run.n], dtype=torch.int32))
    out, lse = run.attend(True)
    assert bool((out[1:] == 7).all()) and bool((out[0, 2:] == 7).all()) and bool((out[0, :2] != 7).all())
    run.begins, run.counts = [run.n - 2, 0, 0], [2, 0, 0]
    run.check(out, lse)


@pytest.mark.gpu
def test_chunks_of_a_prompt_attend_as_the_whole_does():
    run = Run(51, [0], [300], softcap=25.0, window=100).device()
    whole, lse = run.attend(True)
    run.check(whole, lse)
    for begin, count in ((0, 128), (128, 1), (129, 171)):
        q = run.dq[:, begin:begin + count].contiguous()
        out = torch.empty_like(q, dtype=torch.float32)
        run.ctx.attend_rows(q, run.dK, run.dV, torch.tensor([begin], dtype=torch.int32, device="cuda"),
                            torch.tensor([count], dtype=torch.int32, device="cuda"), 1, count, run.scale, out, **run.mods)
        assert float((out - whole[:, begin:begin + count]).abs().max()) <= 2 * float(run.attention()[2].max())


@pytest.mark.gpu
def test_dense_decode_and_a_run_of_one_agree():
    run = Run(61, [777], [1], d=128).device()
    out, _ = run.attend(True)
    dense = torch.empty((1, run.Hq, run.d), device="cuda")
    run.ctx.dense_decode(run.dq[:, 0].contiguous(), run.dK, run.dV, torch.tensor([778], dtype=torch.int32, device="cuda"), 1,
                         run.scale, dense)
    assert bool(((out[:, 0] - dense).abs().cpu() <= 2 * run.attention()[2][:, 0]).all())


@pytest.mark.gpu
def test_streams_graphs_and_repeats():
    """Captured with its masses on a side stream and replayed with new lengths and inputs between eager calls."""
    run = Run(71, [600, 20], [3, 3], page=16, softcap=30.0).device()
    stream = torch.cuda.Stream()
    out = torch.full(run.dq.shape, 7.0, device="cuda")
    lse = torch.full(run.dq.shape[:3], 7.0, device="cuda")
    mass = torch.zeros((2, run.Hkv, run.n), device="cuda")
    torch.cuda.synchronize()
    with sk.Graph.capture(stream) as graph:
        run.ctx.attend_rows(run.dq, run.dK, run.dV, run.dbegin, run.dcount, 2, 3, run.scale, out, lse=lse, stream=stream, **run.mods)
        run.ctx.key_mass(run.dq, run.dK, lse, run.dbegin, run.dcount, 2, 3, run.scale, mass, decay=0.0, stream=stream, **run.mods)
    for begins, counts in (([600, 20], [3, 3]), ([100, 555], [1, 3]), ([0, 601], [2, 0]), ([600, 20], [3, 3])):
        run.dbegin.copy_(torch.tensor(begins, dtype=torch.int32))
        run.dcount.copy_(torch.tensor(counts, dtype=torch.int32))
        run.begins, run.counts = begins, counts
        run.dq.normal_()
        run.q = run.dq.cpu().double()
        out.fill_(7.0)
        lse.fill_(7.0)
        mass.fill_(3.0)
        torch.cuda.synchronize()
        graph.launch()
        torch.cuda.synchronize()
        run.check(out, lse)
        eager, eager_lse = run.attend(True)
        assert torch.equal(eager, out) and torch.equal(eager_lse, lse)
        want, tol = run.masses(torch.full(mass.shape, 3.0, dtype=torch.float64), 0.0, 0, lse.cpu())
        assert bool(((mass.cpu().double() - want).abs() <= tol).all())
    graph.close()


@pytest.mark.gpu
def test_rows_past_four_gigabytes():
    """A cache of 4.8 GB: the last head's last rows lie beyond what 32-bit offsets reach."""
    n, Hkv, d = 1172000, 8, 256
    ctx = sk.Context(sk.make_params(d, Hkv, Hkv, 16, 4, sk.BF16, 1, n, 16))
    K = torch.randn((1, Hkv, n, d), dtype=torch.bfloat16, device="cuda")
    V = torch.randn((1, Hkv, n, d), dtype=torch.bfloat16, device="cuda")
    q = torch.randn((1, 2, Hkv, d), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.zeros((1, 2, Hkv, d), device="cuda"), torch.zeros((1, 2, Hkv), device="cuda")
    mass = torch.zeros((1, Hkv, n), device="cuda")
    begin, count = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (n - 2, 2))
    ctx.attend_rows(q, K, V, begin, count, 1, 2, 1 / 16, out, lse=lse)
    ctx.key_mass(q, K, lse, begin, count, 1, 2, 1 / 16, mass, decay=0.0)
    s = q[0, 1, Hkv - 1].double() @ K[0, Hkv - 1].double().T / 16
    p = torch.softmax(s, -1)
    want = p @ V[0, Hkv - 1].double()
    # sums of n terms in fp32, split and tiled: no chain is longer than n / 128 splits; 2e-5 of sum p |v| covers it
    assert float((out[0, 1, Hkv - 1].double() - want).abs().max()) <= 2e-5 * float((p @ V[0, Hkv - 1].double().abs()).max())
    assert abs(float(lse[0, 1, Hkv - 1]) - float(torch.logsumexp(s, -1))) <= 2e-5
    assert abs(float(mass[0, Hkv - 1].double().sum()) - 2.0) <= 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("mods", range(len(MODS)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("f32", [False, True])
def test_masses_of_runs(f32, shape, mods):
    m = dict(MODS[mods])
    if "prefix" in m:
        m["prefix"] = m["prefix"][: len(SHAPES[shape]["begins"])]
    run = Run(300 + 10 * shape + mods, f32=f32, page=[16, 0, 48][(shape + mods) % 3], **SHAPES[shape], **m).device()
    lse = run.attention()[1].float()
    before = torch.rand((run.B, run.Hkv, run.n), generator=torch.Generator().manual_seed(shape))
    for decay, last in ((0.0, 0), (0.9, 0), (1.0, 7), (0.5, 64)):
        mass = before.cuda()
        run.ctx.key_mass(run.dq, run.dK, lse.cuda(), run.dbegin, run.dcount, run.B, run.R, run.scale, mass, decay=decay,
                         last_rows=last, **run.mods)
        want, tol = run.masses(before.double(), float(np.float32(decay)), last, lse)
        assert float(((mass.cpu().double() - want).abs() - tol).max()) <= 0, (decay, last)
        again = before.cuda()
        run.ctx.key_mass(run.dq, run.dK, lse.cuda(), run.dbegin, run.dcount, run.B, run.R, run.scale, again, decay=decay,
                         last_rows=last, **run.mods)
        assert torch.equal(mass, again)


@pytest.mark.gpu
@pytest.mark.parametrize("G,Hkv,d,f32", [(1, 1, 256, True), (2, 3, 256, False), (8, 2, 64, False), (8, 1, 64, True)])
def test_masses_of_heads_and_widths(G, Hkv, d, f32):
    run = Run(17 * d + G, [250, 3], [37, 90], G=G, Hkv=Hkv, d=d, f32=f32).device()
    lse = run.attention()[1].float()
    mass = torch.full((2, Hkv, run.n), math.nan, device="cuda")
    run.ctx.key_mass(run.dq, run.dK, lse.cuda(), run.dbegin, run.dcount, 2, run.R, run.scale, mass, decay=0.0, **run.mods)
    for b in range(2):
        end = run.begins[b] + run.counts[b]
        want, tol = run.masses(torch.zeros((2, Hkv, run.n), dtype=torch.float64), 0.0, 0, lse)
        assert bool(((mass[b, :, :end].cpu().double() - want[b, :, :end]).abs() <= tol[b, :, :end]).all())
        assert bool(torch.isnan(mass[b, :, end:]).all())
        # every row gives its weight away whole
        assert torch.allclose(mass[b, :, :end].double().sum(-1).cpu(), torch.full((Hkv,), float(run.counts[b] * G), dtype=torch.float64), rtol=1e-4)


@pytest.mark.gpu
def test_masses_ignore_what_is_not_seen():
    run = Run(81, [100], [60], page=16, docs=[120], spare=20)
    run.K[0, :, 160:] = math.nan
    run.K[0, 0, 119] = math.inf                          # seen by the first document's rows alone
    run.table[0, 2] = -5
    run.docs[0, 130] = 4000                              # a row that sees nothing
    run.device()
    lse = run.attention()[1].float()
    lse[0, :20] = 3.0
    lse[0, 30] = -math.inf
    mass = torch.zeros((1, run.Hkv, run.n), device="cuda")
    run.ctx.key_mass(run.dq, run.dK, lse.cuda(), run.dbegin, run.dcount, 1, 60, run.scale, mass, decay=1.0, last_rows=40, **run.mods)
    want, tol = run.masses(torch.zeros((1, run.Hkv, run.n), dtype=torch.float64), 1.0, 40, lse)
    assert bool(torch.isfinite(mass).all())
    assert float(((mass.cpu().double() - want).abs() - tol).max()) <= 0


@pytest.mark.gpu
def test_refusals():
    run = Run(91, [40], [4], page=16).device()
    out, lse = run.attend(True)
    mass = torch.zeros((1, run.Hkv, run.n), device="cuda")
    kw = dict(run.mods)

    def attend(**more):
        a = dict(batch=1, max_rows=4, scale=1.0, **kw)
        a.update(more)
        batch, rows, scale = a.pop("batch"), a.pop("max_rows"), a.pop("scale")
        run.ctx.attend_rows(run.dq, run.dK, run.dV, run.dbegin, run.dcount, batch, rows, scale, out, **a)

    def masses(**more):
        a = dict(batch=1, max_rows=4, scale=1.0, **kw)
        a.update(more)
        batch, rows, scale = a.pop("batch"), a.pop("max_rows"), a.pop("scale")
        run.ctx.key_mass(run.dq, run.dK, lse, run.dbegin, run.dcount, batch, rows, scale, mass, **a)
    for call in (attend, masses):
        for bad in (dict(batch=0), dict(batch=2), dict(max_rows=-1), dict(max_rows=run.n + 1), dict(scale=math.nan),
                    dict(scale=math.inf), dict(softcap=-1.0), dict(softcap=math.inf), dict(softcap=math.nan), dict(window=-3),
                    dict(block_table=None)):
            with pytest.raises(sk.SocketError) as e:
                call(**bad)
            assert e.value.code == sk.EINVAL, bad
        call(max_rows=0)
    for bad in (dict(decay=-0.1), dict(decay=math.nan), dict(last_rows=-1)):
        with pytest.raises(sk.SocketError):
            masses(**bad)
    lib, odd = sk.lib(), run.dq.data_ptr() + 4
    assert lib.socket_attend_rows(run.ctx._h, odd, run.dK.data_ptr(), run.dV.data_ptr(), run.dtable.data_ptr(), run.dbegin.data_ptr(),
                                  run.dcount.data_ptr(), 1, 4, 1.0, None, sk.F32, out.data_ptr(), None, None) == sk.EINVAL
    assert lib.socket_attend_rows(run.ctx._h, run.dq.data_ptr(), run.dK.data_ptr(), run.dV.data_ptr(), run.dtable.data_ptr(),
                                  run.dbegin.data_ptr(), run.dcount.data_ptr(), 1, 4, 1.0, None, 5, out.data_ptr(), None, None) == sk.EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("mods", [dict(), dict(window=300, bias=True), dict(softcap=20.0, prefix=[500, 2, 0], docs=[130, 700])])
def test_whole_prompts_split_over_keys_and_queries(mods, f32, d):
    run = Run(94 + d, [0, 100, 0], [1100, 3, 0], G=1, d=d, f32=f32, **mods).device()
    out, lse = run.attend(True)
    run.check(out, lse)
    before = torch.rand((3, run.Hkv, run.n), generator=torch.Generator().manual_seed(7)).double().float().double()
    want, tol = run.masses(before, 0.5, 0, lse.cpu())
    mass = before.float().cuda()
    run.ctx.key_mass(run.dq, run.dK, lse, run.dbegin, run.dcount, 3, run.R, run.scale, mass, decay=0.5, **run.mods)
    assert float(((mass.cpu().double() - want).abs() - tol).max()) <= 0
    again = before.float().cuda()
    run.ctx.key_mass(run.dq, run.dK, lse, run.dbegin, run.dcount, 3, run.R, run.scale, again, decay=0.5, **run.mods)
    assert torch.equal(mass, again)


@pytest.mark.gpu
def test_caps_and_scales_where_fp32_ends():
    run = Run(92, [40], [4]).device()
    out, lse = run.attend(True)
    mass = torch.zeros((1, run.Hkv, run.n), device="cuda")
    for scale, cap in ((1e31, 0.0), (-1e31, 0.0), (1.0, 1e-39), (1.0, 1e38), (1e20, 1e-20)):
        for call in (lambda: run.ctx.attend_rows(run.dq, run.dK, run.dV, run.dbegin, run.dcount, 1, 4, scale, out, softcap=cap),
                     lambda: run.ctx.key_mass(run.dq, run.dK, lse, run.dbegin, run.dcount, 1, 4, scale, mass, softcap=cap)):
            with pytest.raises(sk.SocketError) as e:
                call()
            assert e.value.code == sk.EINVAL, (scale, cap)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [4, 90])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("cap", [1e30, 1e-30])           # as good as none; every score is the cap or its negative
def test_the_largest_and_the_smallest_cap(cap, f32, rows):
    run = Run(93, [40], [rows], f32=f32, softcap=cap).device()
    run.check(*run.attend(True))


def test_null_arguments_are_refused_without_a_gpu():
    lib = sk.lib()
    assert lib.socket_attend_rows(None, None, None, None, None, None, None, 1, 1, 1.0, None, 1, None, None, None) == sk.EINVAL
    assert lib.socket_key_mass(None, None, None, None, None, None, None, 1, 1, 1.0, None, 1.0, 0, None, None) == sk.EINVAL
    assert lib.socket_evict_select(None, None, None, None, None, 1, 1, None, None, None, None) == sk.EINVAL
    assert lib.socket_evict_rows(*([None] * 3), 1, *([None] * 13)) == sk.EINVAL
