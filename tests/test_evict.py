"""Eviction: the select of the tokens to keep (socket_evict_select) and the move of their rows (socket_evict_rows),
both exact, and the prompt's path through them."""
import math

import numpy as np
import pytest
import torch

import harness
from paper_2602_06283_amd import binding as sk
from paper_2602_06283_amd import workloads as wl


def wanted(mass, length, keep, pool, sink, window, absent=None):
    """Positions kept of one row of masses, ascending."""
    n = max(0, min(length, len(mass)))
    x = mass[:n].astype(np.float64)
    x = np.where(x >= np.finfo(np.float32).min, np.minimum(x, np.finfo(np.float32).max), np.finfo(np.float32).min)
    y = np.array([x[max(0, t - pool // 2):t + pool // 2 + 1].max() for t in range(n)])
    y[:sink] = np.inf
    y[max(0, n - window):] = np.inf
    ok = np.ones(n, bool) if absent is None else ~absent[:n]
    order = np.lexsort((np.arange(n), -y))
    return np.sort(order[ok[order]][:max(0, keep)])


@pytest.mark.gpu
@pytest.mark.parametrize("pool", [1, 3, 7, 11, 255])
@pytest.mark.parametrize("n,page", [(16, 0), (1008, 48), (5008, 0), (50000, 16)])
def test_select_keeps_the_largest_masses(n, page, pool):
    rng = np.random.default_rng(n + pool)
    B, Hkv, k = 4, 2, max(2, n // 5)
    blocks = -(-n // page) if page else 0
    ctx = sk.Context(sk.make_params(64, 2, Hkv, 16, 4, sk.BF16, B, n, k, page, blocks, blocks * B))
    mass = (rng.random((B, Hkv, n)) ** 6).astype(np.float32)
    mass[0, 0, rng.integers(0, n, n // 3)] = 0.25                # many equal
    mass[1, 0, 5], mass[1, 1, 3], mass[1, 1, 7] = math.nan, -math.inf, math.inf
    lens, keep = [n, n - 3, 1, 0], [k, k // 2, k, k]
    if pool == 3:
        keep[1] = 0
    table, absent = None, None
    if page:
        table = rng.permutation(B * blocks).reshape(B, blocks).astype(np.int32)
        table[0, 1] = -1
        absent = np.zeros((B, blocks * page), bool)
        absent[0, page:2 * page] = True
    for sink, window in ((0, 0), (2, 5)):
        ctx.set_forced_tokens(sink, window)
        scores = torch.full((B, Hkv, n), math.nan, device="cuda")
        idx = torch.full((B, Hkv, k), -7, dtype=torch.int32, device="cuda")
        count = torch.full((B, Hkv), -7, dtype=torch.int32, device="cuda")
        ctx.evict_select(torch.from_numpy(mass).cuda(), harness.i32(lens), harness.i32(keep), B, scores, idx, count, pool=pool,
                         block_table=None if table is None else torch.from_numpy(table).cuda())
        got, c = idx.cpu().numpy(), count.cpu().numpy()
        for b in range(B):
            for h in range(Hkv):
                w = wanted(mass[b, h], lens[b], keep[b], pool, sink, window, None if absent is None else absent[b])
                assert c[b, h] == len(w)
                assert (got[b, h, :len(w)] == w).all() and (got[b, h, len(w):] == -1).all(), (b, h)


IDS = [(64, 8), (16, 8), (24, 5), (100, 8), (60, 10), (16, 9), (128, 10), (20, 12), (128, 4), (300, 2)]


class Cache:
    """K, V, ids, norms and masses of a batch, contiguous or paged, every byte of it drawn."""

    def __init__(self, seed, L, P, d=64, f32=False, B=2, Hkv=2, n=336, page=0, k=None):
        g = torch.Generator().manual_seed(seed)
        self.L, self.P, self.B, self.Hkv, self.n, self.page, self.d = L, P, B, Hkv, n, page, d
        dt = torch.float32 if f32 else torch.bfloat16
        blocks = n // page if page else 0
        lead = (B * blocks * 2, Hkv) if page else (B, Hkv)
        rows = page or n
        self.K, self.V = (torch.randn(lead + (rows, d), generator=g).to(dt).cuda() for _ in range(2))
        nat = torch.randint(0, 1 << P, lead + (rows, L), generator=g).numpy().astype(harness.code_dtype(P))
        self.codes = harness.rows_to_device(harness.codes_from_natural(nat, L, harness.code_dtype(P), P=P), L, P)
        self.norms, self.mass = (torch.rand((B, Hkv, n), generator=g).cuda() for _ in range(2))
        self.table = self.table2 = None
        if page:
            perm = torch.randperm(B * blocks * 2, generator=g).to(torch.int32)
            self.table, self.table2 = perm[: B * blocks].view(B, blocks).cuda(), perm[B * blocks:].view(B, blocks).cuda()
        self.k = k or n // 2
        self.ctx = sk.Context(sk.make_params(d, Hkv, Hkv, L, P, sk.F32 if f32 else sk.BF16, B, n, self.k, page, blocks, B * blocks * 2))
        self.idx = torch.full((B, Hkv, self.k), -1, dtype=torch.int32)
        self.count = torch.zeros((B, Hkv), dtype=torch.int32)
        for b in range(B):
            for h in range(Hkv):
                c = [self.k, self.k // 3, 1, 0][(b * Hkv + h) % 4]
                self.idx[b, h, :c] = torch.randperm(n, generator=g)[:c].sort().values
                self.count[b, h] = c

    def natural(self, x, table, ids=False):
        """In token order on the host: [B, Hkv, n, ...]; ids [.., L]."""
        x = x.cpu()
        if ids:
            x = torch.from_numpy(harness.codes_to_natural(harness.rows_from_device(x, self.L, self.P), self.L, P=self.P).astype(np.int32))
        elif x.dtype == torch.bfloat16:
            x = x.float()
        if table is not None:
            x = x[table.cpu().long()].transpose(1, 2)
            x = x.reshape((self.B, self.Hkv, self.n) + x.shape[4:])
        return x.numpy()

    def all(self, tensors, table):
        K, V, codes, norms, mass = tensors
        return [self.natural(K, table), self.natural(V, table), self.natural(codes, table, ids=True), norms.cpu().numpy(), mass.cpu().numpy()]

    def move(self, out, table, table_out, **more):
        self.ctx.evict_rows(self.idx.cuda(), self.count.cuda(), self.B, self.K, self.V, out[0], out[1], codes=self.codes, codes_out=out[2],
                            vnorm=self.norms, vnorm_out=out[3], mass=self.mass, mass_out=out[4], block_table=table,
                            block_table_out=table_out, **more)

    def check(self, before, after, untouched):
        """after = before's kept rows at the front, `untouched` behind."""
        for x, y, z in zip(before, after, untouched):
            for b in range(self.B):
                for h in range(self.Hkv):
                    c = int(self.count[b, h])
                    assert (y[b, h, :c] == x[b, h][self.idx[b, h, :c].numpy()]).all(), (b, h)
                    assert (y[b, h, c:] == z[b, h, c:]).all(), (b, h)


@pytest.mark.gpu
@pytest.mark.parametrize("page", [0, 48])
@pytest.mark.parametrize("L,P", IDS)
def test_move_to_other_tensors_and_in_place(L, P, page):
    c = Cache(L + P, L, P, page=page)
    before = c.all((c.K, c.V, c.codes, c.norms, c.mass), c.table)
    out = [torch.zeros_like(x) for x in (c.K, c.V, c.codes, c.norms, c.mass)]
    zeros = c.all(out, c.table2)
    c.move(out, c.table, c.table2)
    c.check(before, c.all(out, c.table2), zeros)
    assert all((x == y).all() for x, y in zip(before, c.all((c.K, c.V, c.codes, c.norms, c.mass), c.table)))
    same = (c.K, c.V, c.codes, c.norms, c.mass)
    c.move(same, c.table, c.table)
    c.check(before, c.all(same, c.table), before)


@pytest.mark.gpu
@pytest.mark.parametrize("d,f32", [(64, True), (128, False), (128, True), (256, False), (256, True)])
def test_move_of_wide_rows(d, f32):
    for page in (0, 16):
        c = Cache(d, 64, 8, d=d, f32=f32, page=page, n=208)
        before = c.all((c.K, c.V, c.codes, c.norms, c.mass), c.table)
        out = [torch.zeros_like(x) for x in (c.K, c.V, c.codes, c.norms, c.mass)]
        zeros = c.all(out, c.table2)
        c.move(out, c.table, c.table2)
        c.check(before, c.all(out, c.table2), zeros)
        same = (c.K, c.V, c.codes, c.norms, c.mass)
        c.move(same, c.table, c.table)
        c.check(before, c.all(same, c.table), before)


@pytest.mark.gpu
def test_move_in_place_over_many_passes():
    """More rows than a pass of the in-place move holds, in rows of 64 ids and of 20 bytes."""
    for L, P, page in ((64, 8, 0), (16, 10, 16)):
        c = Cache(3, L, P, B=1, Hkv=4, n=20000, page=page, k=15001)
        before = c.all((c.K, c.V, c.codes, c.norms, c.mass), c.table)
        same = (c.K, c.V, c.codes, c.norms, c.mass)
        c.move(same, c.table, c.table)
        c.check(before, c.all(same, c.table), before)


@pytest.mark.gpu
def test_move_in_place_under_a_copy_of_the_block_table():
    c = Cache(17, 64, 8, B=1, Hkv=2, n=6000, page=48, k=5001)
    before = c.all((c.K, c.V, c.codes, c.norms, c.mass), c.table)
    same = (c.K, c.V, c.codes, c.norms, c.mass)
    c.move(same, c.table, c.table.clone())
    c.check(before, c.all(same, c.table), before)


@pytest.mark.gpu
def test_move_within_the_same_pools_and_without_the_optional_arrays():
    c = Cache(9, 64, 8, page=16)
    before = c.all((c.K, c.V, c.codes, c.norms, c.mass), c.table)
    norms, mass = c.norms.clone(), c.mass.clone()
    # other blocks of the same pools; the float arrays, by sequence, in place
    behind = c.all((c.K, c.V, c.codes, norms, mass), c.table2)
    c.move((c.K, c.V, c.codes, c.norms, c.mass), c.table, c.table2)
    c.check(before, c.all((c.K, c.V, c.codes, c.norms, c.mass), c.table2), behind)
    K, V = torch.zeros_like(c.K), torch.zeros_like(c.V)
    c.ctx.evict_rows(c.idx.cuda(), c.count.cuda(), c.B, c.K, c.V, K, V, block_table=c.table, block_table_out=c.table2)
    got = c.natural(K, c.table2)
    for b in range(c.B):
        for h in range(c.Hkv):
            m = int(c.count[b, h])
            assert (got[b, h, :m] == before[0][b, h][c.idx[b, h, :m].numpy()]).all() and (got[b, h, m:] == 0).all()


@pytest.mark.gpu
def test_entries_and_blocks_that_are_not_there_are_skipped():
    c = Cache(13, 60, 10, page=16)
    before = c.all((c.K, c.V, c.codes, c.norms, c.mass), c.table)
    c.idx[0, 0, 3], c.idx[0, 0, 9] = -1, c.n
    c.count[0, 0] = c.k + 1000                          # (no more than the row holds)
    gone, hole = c.table.clone(), c.table2.clone()
    gone[0, 7], hole[0, 2] = -1, 10 ** 6
    out = [torch.zeros_like(x) for x in (c.K, c.V, c.codes, c.norms, c.mass)]
    c.move(out, gone, hole)
    after = c.all(out, c.table2)
    for x, y in zip(before, after):
        for j in range(c.k):
            t = int(c.idx[0, 0, j])
            there = 0 <= t < c.n and t // 16 != 7 and j // 16 != 2
            assert (y[0, 0, j] == (x[0, 0, t] if there else 0)).all(), j


@pytest.mark.gpu
@pytest.mark.parametrize("pool", [1, 5])
def test_tokens_that_are_always_kept_come_before_infinite_masses(pool):
    n = 64
    ctx = sk.Context(sk.make_params(64, 1, 1, 16, 4, sk.BF16, 1, n, 8))
    ctx.set_forced_tokens(0, 3)
    mass = torch.ones((1, 1, n), device="cuda")
    mass[0, 0, :40] = math.inf
    scores, idx, count = torch.empty_like(mass), torch.full((1, 1, 8), -7, dtype=torch.int32, device="cuda"), harness.i32([[0]])
    ctx.evict_select(mass, harness.i32([n]), harness.i32([5]), 1, scores, idx, count, pool=pool)
    assert idx[0, 0].tolist() == [0, 1, 61, 62, 63, -1, -1, -1] and count.item() == 5


@pytest.mark.gpu
def test_refusals():
    c = Cache(15, 64, 8, page=16)
    out = [torch.zeros_like(x) for x in (c.K, c.V, c.codes, c.norms, c.mass)]
    idx, count = c.idx.cuda(), c.count.cuda()
    for more in (dict(codes=c.codes), dict(codes_out=out[2]), dict(vnorm=c.norms), dict(mass_out=out[4])):
        with pytest.raises(sk.SocketError) as e:
            c.ctx.evict_rows(idx, count, c.B, c.K, c.V, out[0], out[1], block_table=c.table, block_table_out=c.table2, **more)
        assert e.value.code == sk.EINVAL
    for table, table_out, batch in ((None, c.table2, 2), (c.table, None, 2), (c.table, c.table2, 3), (c.table, c.table2, 0)):
        with pytest.raises(sk.SocketError):
            c.ctx.evict_rows(idx, count, batch, c.K, c.V, out[0], out[1], block_table=table, block_table_out=table_out)
    assert sk.lib().socket_evict_rows(c.ctx._h, idx.data_ptr(), count.data_ptr(), c.B, c.K.data_ptr() + 2, c.V.data_ptr(), None, None, None,
                                      c.table.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), None, None, None, c.table2.data_ptr(),
                                      None) == sk.EINVAL
    lens, scores = harness.i32([c.n] * 2), torch.empty_like(c.mass)
    for pool, into, batch, table in ((0, scores, 2, c.table), (2, scores, 2, c.table), (257, scores, 2, c.table), (3, c.mass, 2, c.table),
                                     (3, scores, 3, c.table), (3, scores, 2, None)):
        with pytest.raises(sk.SocketError) as e:
            c.ctx.evict_select(c.mass, lens, lens, batch, into, idx, count, pool=pool, block_table=table)
        assert e.value.code == sk.EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("L,P,page,f32", [(64, 8, 0, False), (60, 10, 16, False), (32, 8, 16, True)])
def test_a_prompt_attended_evicted_and_decoded(L, P, page, f32):
    """The calls together, as a serving program makes them, on one stream and nothing waited for: attend the prompt,
    hash its keys, gather the masses of its last rows, evict in place, decode over what is left.  The ids that moved
    are those that hashing the moved keys gives, and a decode step on the evicted cache is the step on a cache that
    was built from the kept rows."""
    layer = wl.make_layer(77, B=2, Hq=8, Hkv=2, d=128, n=1536, L=L, P=P, k=64, kv_dtype=wl.F32 if f32 else wl.BF16)
    B, Hkv, n, keep, prompt = 2, 2, layer.n, [300, 257], [1500, 1111]
    blocks = n // page if page else 0
    ctx = harness.make_ctx(layer, max_k=512, page=page, max_blocks=blocks, num_blocks=B * blocks)
    K, V, W = (harness.dev(x, layer.kv_dtype) for x in (layer.K, layer.V, layer.W))
    table = None
    if page:
        table = torch.randperm(B * blocks).to(torch.int32).view(B, blocks).cuda()
        pooled = [torch.zeros((B * blocks, Hkv, page, 128), dtype=K.dtype, device="cuda") for _ in range(2)]
        for pool, x in zip(pooled, (K, V)):
            pool[table.view(-1).long()] = x.view(B, Hkv, blocks, page, 128).transpose(1, 2).reshape(pool.shape)
        K, V = pooled
    g = torch.Generator().manual_seed(5)
    q = torch.randn((B, n, 8, 128), generator=g).to(K.dtype).cuda()
    lead = (B * blocks,) if page else (B,)
    codes = harness.new_codes(lead + (Hkv,), page or n, L, P)
    zero, lens, kk = harness.i32([0, 0]), harness.i32(prompt), harness.i32(keep)
    out = torch.zeros((B, n, 8, 128), device="cuda")
    lse = torch.zeros((B, n, 8), device="cuda")
    mass, scores, norms = (torch.zeros((B, Hkv, n), device="cuda") for _ in range(3))
    idx, count = torch.zeros((B, Hkv, 512), dtype=torch.int32, device="cuda"), torch.zeros((B, Hkv), dtype=torch.int32, device="cuda")
    K0, V0 = K.clone(), V.clone()
    ctx.set_forced_tokens(4, 32)
    ctx.attend_rows(q, K, V, zero, lens, B, n, 128 ** -0.5, out, lse=lse, block_table=table)
    ctx.hash_keys(K, W, zero, lens, B, n, codes, block_table=table)
    ctx.value_norms(V, zero, lens, B, n, norms, block_table=table)
    ctx.key_mass(q, K, lse, zero, lens, B, n, 128 ** -0.5, mass, decay=0.0, last_rows=64, block_table=table)
    ctx.evict_select(mass, lens, kk, B, scores, idx, count, pool=5, block_table=table)
    ctx.evict_rows(idx, count, B, K, V, K, V, codes=codes, codes_out=codes, vnorm=norms, vnorm_out=norms, mass=mass, mass_out=mass,
                   block_table=table, block_table_out=table)
    left = count[:, 0].contiguous()
    again = codes.clone()
    ctx.hash_keys(K, W, zero, left, B, 512, again, block_table=table)
    assert count.cpu().tolist() == [[keep[0]] * 2, [keep[1]] * 2]
    for b in range(B):                                  # forced tokens are there, and positions ascend
        for h in range(Hkv):
            kept = idx[b, h, :keep[b]].cpu().numpy()
            assert (np.diff(kept) > 0).all() and (kept[:4] == np.arange(4)).all() and (kept[-32:] == np.arange(prompt[b] - 32, prompt[b])).all()
    assert torch.equal(codes, again)

    def token_order(x):
        return x if table is None else x[table.long()].transpose(1, 2).reshape(B, Hkv, n, 128)
    K1, V1, Ks, Vs = (token_order(x) for x in (K, V, K0, V0))
    for b in range(B):
        for h in range(Hkv):
            kept = idx[b, h, :keep[b]].long()
            assert torch.equal(K1[b, h, :keep[b]], Ks[b, h][kept]) and torch.equal(V1[b, h, :keep[b]], Vs[b, h][kept])
            # (value norms: the same rows, the same sums)
            assert torch.allclose(norms[b, h, :keep[b]], V1[b, h, :keep[b]].float().norm(dim=-1), rtol=1e-6)
    # a decode step behind the eviction, and the same step on a context and cache of its own
    q1 = torch.randn((B, 8, 128), generator=g).to(K.dtype).cuda()
    results = []
    for fresh in (False, True):
        c2 = harness.make_ctx(layer, max_k=512, page=page, max_blocks=blocks, num_blocks=B * blocks) if fresh else ctx
        if fresh:
            c2.set_forced_tokens(4, 32)
            K, V = K.clone(), V.clone()
            codes = harness.new_codes(lead + (Hkv,), page or n, L, P)
            c2.hash_keys(K, W, zero, left, B, 512, codes, block_table=table)
        y = torch.zeros((B, 8, 128), device="cuda")
        c2.decode_step(q1, K, V, codes, W, 0.5, left, harness.i32([64, 64]), B, 1.0, scores, idx, count, y, block_table=table)
        results.append((y, idx.clone(), count.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*results))
