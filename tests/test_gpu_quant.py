"""The 8-bit KV cache on the GPU against its fp64 oracle: the store, attention
over the cache, key bounds and the selection of blocks."""

import math

import numpy as np
import pytest
import torch

import oracle as O
from oracle import quant_oracle as Q
from paper_2602_08329_amd import binding as B
from tests.quant_tolerance import assert_attention

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4 = torch.float8_e4m3fn
I32 = torch.int32


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


class Cache:
    """A seeded 8-bit cache on the host (NumPy) and its copy on the GPU.  Rows at
    and behind a sequence's length, and unused pages, hold NaN bytes and NaN
    scales of blocks no token lies in."""

    def __init__(self, lens, hq, hkv, d, bs=16, paged=False, dtype="bf16", seed=0, spread=3.0,
                 fill=True, cap=None):
        rng = np.random.default_rng(seed)
        self.lens, self.hq, self.hkv, self.d, self.bs, self.paged = lens, hq, hkv, d, bs, paged
        self.dtype = torch.float32 if dtype == "f32" else torch.bfloat16
        n_cap = max(max(lens), 1) if cap is None else cap
        self.nb = -(-n_cap // bs)
        Bn = len(lens)
        self.pages = Bn * self.nb + 3 if paged else 0
        blocks = self.pages * hkv if paged else Bn * hkv * self.nb
        self.table = rng.permutation(self.pages)[: Bn * self.nb].reshape(Bn, self.nb) if paged else None
        self.raw = {x: np.full((blocks, bs, d), 127, np.uint8) for x in "kv"}
        self.scale = {x: np.full(blocks, np.nan, np.float32) for x in "kv"}
        if fill:
            for b, n in enumerate(lens):
                for g in range(hkv):
                    for j in range(-(-n // bs)):
                        i, r = self.block(b, g, j), min(bs, n - j * bs)
                        for x in "kv":
                            v = rng.integers(0, 127, (r, d)) * 1 + 128 * rng.integers(0, 2, (r, d))
                            self.raw[x][i, :r] = v
                            # K: unit logits whatever the scale's spread
                            s = 2.0 ** rng.uniform(-spread, spread)
                            self.scale[x][i] = s / (200 if x == "k" else 100)
        shape = (self.pages, hkv, bs, d) if paged else (Bn, hkv, self.nb * bs, d)
        sshape = (self.pages, hkv) if paged else (Bn, hkv, self.nb)
        dev = {x: torch.tensor(self.raw[x]).to(DEV).view(E4).view(shape) for x in "kv"}
        dsc = {x: torch.tensor(self.scale[x]).to(DEV).view(sshape) for x in "kv"}
        self.dev, self.dsc = dev, dsc
        self.seq = torch.tensor(lens, dtype=I32, device=DEV)
        self.dtable = torch.tensor(self.table, dtype=I32, device=DEV) if paged else None
        self.kv = B.QuantKV(dev["k"], dev["v"], dsc["k"], dsc["v"], self.seq, n_cap, hq, self.dtable,
                            dtype=self.dtype)
        q = rng.standard_normal((Bn, hq, d))
        self.q = torch.tensor(q, dtype=torch.float32).to(self.dtype).to(DEV)
        self.scale_q = 1 / math.sqrt(d)

    def block(self, b, g, j):
        if self.paged:
            return int(self.table[b, j]) * self.hkv + g
        return (b * self.hkv + g) * self.nb + j

    def values(self, x, b, g, n):
        """Rows [0, n) of a unit in fp64."""
        rows = [Q.TABLE[self.raw[x][self.block(b, g, j)]] * float(self.scale[x][self.block(b, g, j)])
                for j in range(-(-n // self.bs))]
        return np.concatenate(rows)[:n] if rows else np.zeros((0, self.d))

    def outputs(self):
        Bn = len(self.lens)
        return (torch.full((Bn, self.hq, self.d), 7.0, device=DEV),
                torch.full((Bn, self.hq), 7.0, device=DEV))

    def workspace(self, dense, cap=0):
        """Exactly the bytes asked for, followed by bytes that must stay."""
        op = B.PRHS_OP_QUANT_DENSE_ATTN if dense else B.PRHS_OP_QUANT_SPARSE_ATTN
        n = B.prhs_workspace_size(op, self.kv, None, cap)
        self.ws_all = torch.full((n + 256,), 255, dtype=torch.uint8, device=DEV)
        return self.ws_all[:n]

    def check(self, y, lse, attended, some=None):
        """attended(b, g): positions, of the units `some` (all by default)."""
        assert (self.ws_all[-256:] == 255).all()
        y, lse = y.double().cpu().numpy(), lse.double().cpu().numpy()
        q = self.q.double().cpu().numpy()
        G = self.hq // self.hkv
        for b in range(len(self.lens)):
            for g in range(self.hkv):
                if some is not None and (b, g) not in some:
                    continue
                S = np.asarray(attended(b, g), dtype=np.int64)
                K, V = (self.values(x, b, g, self.lens[b])[S] for x in "kv")
                for h in range(g * G, (g + 1) * G):
                    if not len(S):
                        assert (y[b, h] == 0).all() and lse[b, h] == -math.inf
                        continue
                    yr, lr = O.dense_attention(q[b, h], K, V, self.scale_q)
                    assert_attention(y[b, h], lse[b, h], yr, lr, q[b, h], K, V, self.scale_q, (b, h))


def dense(c):
    y, lse = c.outputs()
    B.prhs_quant_dense_decode_attn(c.kv, c.q, c.scale_q, y, lse, c.workspace(True))
    return y, lse


def pack(sets, batch, hkv, cap, fill=-7):
    idx = torch.full((batch, hkv, cap), fill, dtype=I32)
    ln = torch.zeros(batch, hkv, dtype=I32)
    for (b, g), S in sets.items():
        idx[b, g, : len(S)] = torch.tensor(list(S), dtype=I32)
        ln[b, g] = len(S)
    return idx.to(DEV), ln.to(DEV)


HEADS = [(1, 1), (2, 2), (6, 2), (5, 1), (8, 1), (18, 2), (16, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,bs,paged", [(128, 16, True), (64, 16, False), (128, 64, False), (64, 128, True), (128, 32, True)])
def test_dense_lengths_around_tiles_and_blocks(d, bs, paged, dtype):
    lens = (0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300)
    hq, hkv = HEADS[(d + bs) % len(HEADS)]
    c = Cache(lens, hq, hkv, d, bs, paged, dtype, seed=d + bs)
    c.check(*dense(c), lambda b, g: range(lens[b]))


@pytest.mark.parametrize("hq,hkv", HEADS)
def test_dense_head_groups(hq, hkv):
    lens = (200, 77)
    for d, dtype in ((128, "bf16"), (64, "f32")):
        c = Cache(lens, hq, hkv, d, seed=hq)
        c.check(*dense(c), lambda b, g: range(lens[b]))


@pytest.mark.parametrize("lens,hq,hkv,d,paged,dtype", [
    ((9001,), 4, 1, 128, True, "bf16"),            # one unit in many splits
    ((5000, 4999, 33, 2500), 8, 2, 64, False, "bf16"),
    ((2048, 2049), 16, 1, 128, False, "f32"),
    (tuple(700 - 3 * i for i in range(40)), 8, 8, 64, True, "bf16"),    # 320 units
    ((70001,), 2, 1, 64, True, "bf16"),            # as many splits as the rows' root allows
    (tuple(2000 - 7 * i for i in range(96)), 2, 1, 128, False, "bf16"),   # two workgroups a CU
    (tuple(8001 - 50 * i for i in range(140)), 1, 1, 64, False, "f32"),   # three splits
    (tuple(4001 - 9 * i for i in range(270)), 1, 1, 64, True, "bf16"),    # four
    ((7, 0, 3), 32, 2, 128, True, "bf16"),         # more waves than tiles
])
def test_dense_splits(lens, hq, hkv, d, paged, dtype):
    c = Cache(lens, hq, hkv, d, 16, paged, dtype, seed=lens[0])
    some = {(b, g) for b in (0, 1, len(lens) // 2, len(lens) - 1) for g in (0, hkv - 1) if b < len(lens)}
    c.check(*dense(c), lambda b, g: range(lens[b]), some)


@pytest.mark.parametrize("paged", [False, True])
def test_dense_long_streams_of_many_units(paged):
    # more units than CUs, streams that are not split: longest first, eight waves
    lens = tuple(8300 if b == 97 else 5000 if b == 3 else 0 if b == 40 else 1 + b % 50 for b in range(260))
    c = Cache(lens, 2, 1, 64, 16, paged, "bf16", seed=12)
    c.check(*dense(c), lambda b, g: range(lens[b]))


@pytest.mark.parametrize("spread", [0.0, 10.0])
def test_scales_far_apart(spread):
    # block scales of V over a factor of 2^20: weights of the smaller blocks keep
    # 2^-32 of the largest one's
    c = Cache((500, 40), 4, 2, 128, 16, True, "bf16", seed=3, spread=spread)
    for x in "k":   # logits stay moderate
        c.scale[x][:] = np.where(np.isnan(c.scale[x]), np.nan, np.float32(1 / 300))
        c.dsc[x].copy_(torch.tensor(c.scale[x]).view(c.dsc[x].shape))
    c.check(*dense(c), lambda b, g: range(c.lens[b]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,bs,paged,cap", [(128, 16, True, 40), (64, 32, False, 600), (128, 64, True, 1500), (128, 128, False, 3000)])
def test_sparse_sets(d, bs, paged, cap, dtype):
    # entries outside the sequence and empty sets; a set longer than its capacity
    # says; entries in any order, one of them twice counts twice
    rng = np.random.default_rng(cap)
    lens = (cap * 2, 1, 5, cap // 2 + 1)
    hq, hkv = 8, 2
    c = Cache(lens, hq, hkv, d, bs, paged, dtype, seed=cap + d)
    sets, want = {}, {}
    for b, n in enumerate(lens):
        for g in range(hkv):
            S = rng.permutation(n)[: int(rng.integers(0, min(n, cap) + 1))]
            if (b, g) == (0, 0):
                S = rng.permutation(n)[:cap]
            if (b, g) == (0, 1):
                S = np.concatenate([S[: cap - 4], [-1, n, 1 << 21, -(1 << 30)]])
            if (b, g) == (2, 0):
                S = np.array([], np.int64)
            if (b, g) == (2, 1):
                S = np.array([1 << 21, -5])
            sets[b, g] = S
            want[b, g] = [p for p in S if 0 <= p < n]
    idx, ln = pack(sets, len(lens), hkv, cap)
    ln[0, 0] = cap + 1000
    y, lse = c.outputs()
    B.prhs_quant_sparse_decode_attn(c.kv, c.q, idx, ln, c.scale_q, y, lse, c.workspace(False, cap))
    c.check(y, lse, lambda b, g: want[b, g])


@pytest.mark.parametrize("d,paged,cap", [(128, True, 100), (64, False, 900)])
def test_reuse_tail(d, paged, cap):
    rng = np.random.default_rng(cap)
    lens, anchors = (cap + 50, 20, 7, cap), (cap + 43, 20, 0, cap + 5)
    c = Cache(lens, 6, 2, d, 16, paged, "bf16", seed=cap)
    sets, want = {}, {}
    for b, n in enumerate(lens):
        n0 = min(anchors[b], n)
        for g in range(2):
            S = np.sort(rng.permutation(n)[: cap // 2])
            sets[b, g], want[b, g] = S, [p for p in S if p < n0] + list(range(n0, n))
    idx, ln = pack(sets, len(lens), 2, cap)
    a = torch.tensor(anchors, dtype=I32, device=DEV)
    y, lse = c.outputs()
    B.prhs_quant_reuse_decode_attn(c.kv, c.q, idx, ln, a, c.scale_q, y, lse, c.workspace(False, cap))
    c.check(y, lse, lambda b, g: want[b, g])


def test_pool_rows_sides_and_window():
    rng = np.random.default_rng(4)
    lens, hkv, cap = (400, 90), 2, 120
    c = Cache(lens, 4, hkv, 128, 16, True, "bf16", seed=6)
    pool = [np.sort(rng.permutation(90)[:50]) for _ in range(5)]
    idx = torch.zeros(5, cap, dtype=I32)
    for r, S in enumerate(pool):
        idx[r, :50] = torch.tensor(S)
    plen = torch.full((5,), 50, dtype=I32, device=DEV)
    rows, tails, gate = [3, 9, 0, 4], [395, 390, 90, 60], [-1, 2, 1, -1]
    rows_d, tails_d, gate_d = (torch.tensor(x, dtype=I32, device=DEV) for x in (rows, tails, gate))
    ps = B.psaw(3, 4, 1, 0.5, 1.0, 8)

    def want(b, g, window):
        u, n = b * hkv + g, lens[b]
        if rows[u] >= 5:
            return []
        S = [p for p in pool[rows[u]] if p < tails[u]] + list(range(min(tails[u], n), n))
        first = B.prhs_psaw_first_visible(ps, n)
        return [p for p in S if not window or p < 8 or p >= first]

    for window in (False, True):
        y, lse = c.outputs()
        for side in (B.PRHS_UNITS_RETRIEVING, B.PRHS_UNITS_SHARING):
            B.prhs_quant_pool_decode_attn(c.kv, c.q, idx.to(DEV), plen, rows_d, tails_d, c.scale_q, y, lse,
                                          c.workspace(False, cap), psaw=ps if window else None,
                                          unit_gate=gate_d, units_side=side)
            if side == B.PRHS_UNITS_RETRIEVING:   # the others are left as they are
                assert (y[0, 2:] == 7).all() and (y[1, :2] == 7).all() and not (y[0, :2] == 7).any()
        c.check(y, lse, lambda b, g: want(b, g, window))


def test_empty_pool_and_empty_sets():
    # no row of the pool, no entry of a set: every output is that of no tokens
    import ctypes
    c = Cache((60, 40), 4, 2, 64, 16, True, "bf16", seed=7)
    i = torch.zeros(4, 8, dtype=I32, device=DEV)
    tail = torch.full((4,), 100, dtype=I32, device=DEV)
    ptr = [ctypes.c_void_p(t.data_ptr()) for t in (c.q, i, tail, i, tail)]
    for call in ("pool", "sparse"):
        y, lse = c.outputs()
        ws = c.workspace(False, 8)
        o = [ctypes.c_void_p(t.data_ptr()) for t in (y, lse, ws)]
        L, st = B.lib(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        if call == "pool":
            B.check(L.prhs_quant_pool_decode_attn(ctypes.byref(c.kv.quant), ptr[0], ptr[1], ptr[2], 0, 8, ptr[3], ptr[4],
                                                  None, 0, None, 0.1, *o, ws.numel(), st))
        else:
            B.check(L.prhs_quant_sparse_decode_attn(ctypes.byref(c.kv.quant), ptr[0], ptr[1], ptr[2], 0, 0.1, *o,
                                                    ws.numel(), st))
        assert (y == 0).all() and (lse == -math.inf).all()


def test_pages_outside_the_pool_and_lengths_beyond_the_bound():
    lens = (100, 64)
    c = Cache(lens, 4, 2, 128, 16, True, "bf16", seed=8)
    t = c.dtable.clone()
    t[0, 2], t[0, 6], t[1, 0] = -1, c.pages, 1 << 30
    c.dtable.copy_(t)
    y, lse = c.outputs()
    B.prhs_quant_dense_decode_attn(c.kv, c.q, c.scale_q, y, lse, c.workspace(True))
    left = ([p for p in range(100) if p // 16 not in (2, 6)], list(range(16, 64)))
    c.check(y, lse, lambda b, g: left[b])
    # a length above max_seq_len counts as max_seq_len, a negative one as none
    c.seq.copy_(torch.tensor([1000, -3], dtype=I32))
    y, lse = c.outputs()
    B.prhs_quant_dense_decode_attn(c.kv, c.q, c.scale_q, y, lse, c.workspace(True))
    c.lens = (100, 0)
    c.check(y, lse, lambda b, g: left[b] if b == 0 else [])


def test_no_lse_and_another_stream():
    c = Cache((500, 60), 8, 2, 128, 16, True, "bf16", seed=9)
    y0, _ = dense(c)
    s = torch.cuda.Stream()
    y1, _ = c.outputs()
    ws = c.workspace(True)
    s.wait_stream(torch.cuda.current_stream())
    B.prhs_quant_dense_decode_attn(c.kv, c.q, c.scale_q, y1, None, ws, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y0, y1)


# ---- the store --------------------------------------------------------------------

class Store:
    """A cache that tokens are stored into, on both sides."""

    def __init__(self, batch, hkv, d, bs, paged, dtype, cap, seed, bounds=True):
        self.c = Cache((0,) * batch, hkv, hkv, d, bs, paged, dtype, seed=seed, fill=False, cap=cap)
        self.rng = np.random.default_rng(seed + 1)
        self.n = [0] * batch
        c = self.c
        blocks = len(c.scale["k"])
        self.lo, self.hi = np.full((blocks, d), 9.0), np.full((blocks, d), -9.0)
        sh = (c.pages, hkv, d) if paged else (batch, hkv, c.nb, d)
        self.dlo, self.dhi = (torch.tensor(x, dtype=c.dtype, device=DEV).view(sh) for x in (self.lo, self.hi))
        self.bounds = B.BlockBounds(c.kv, self.dlo, self.dhi) if bounds else None

    def tokens(self, T, wide=4.0):
        c = self.c
        x = self.rng.standard_normal((2, len(self.n), c.hkv, T, c.d)) * 2.0 ** self.rng.uniform(-wide, wide, (2, len(self.n), c.hkv, T, 1))
        return [torch.tensor(y, dtype=torch.float32).to(c.dtype) for y in x]

    def store(self, k, v, new=None, dropped=()):
        """new: tokens of each sequence (all of k's by default)."""
        c, T = self.c, k.shape[2]
        new = [T] * len(self.n) if new is None else new
        for b, t in enumerate(new):
            first, self.n[b] = self.n[b], self.n[b] + t
            for g in range(c.hkv):
                for j in range(first // c.bs, -(-self.n[b] // c.bs)):
                    a, z = max(first, j * c.bs), min(self.n[b], (j + 1) * c.bs)
                    if z <= a or (b, j) in dropped:
                        continue
                    i, r0 = c.block(b, g, j), a - j * c.bs
                    for x, src in (("k", k), ("v", v)):
                        xs = src[b, g, a - first: z - first].double().numpy()
                        c.raw[x][i, : z - j * c.bs], c.scale[x][i] = Q.store_block(c.raw[x][i, :r0], c.scale[x][i], xs)
                        if x == "k" and self.bounds is not None:
                            lo, hi = Q.block_bounds(xs)
                            old = r0 > 0
                            self.lo[i] = np.minimum(lo, self.lo[i]) if old else lo
                            self.hi[i] = np.maximum(hi, self.hi[i]) if old else hi
        c.seq.copy_(torch.tensor(self.n, dtype=I32))
        nl = torch.tensor(new, dtype=I32, device=DEV)
        B.prhs_quant_store(c.kv, k.to(DEV), v.to(DEV), nl, self.bounds)

    def check(self):
        c = self.c
        for x in "kv":
            got = c.dev[x].view(torch.uint8).cpu().numpy().reshape(c.raw[x].shape)
            nan = (got & 127) == 127
            want_nan = (c.raw[x] & 127) == 127
            assert np.array_equal(nan, want_nan) and np.array_equal(got[~nan], c.raw[x][~nan])
            assert np.array_equal(c.dsc[x].cpu().numpy().ravel(), c.scale[x], equal_nan=True)
        assert np.array_equal(self.dlo.double().cpu().numpy().reshape(self.lo.shape), self.lo)
        assert np.array_equal(self.dhi.double().cpu().numpy().reshape(self.hi.shape), self.hi)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,bs,paged", [(128, 16, True), (64, 16, False), (64, 32, True), (128, 64, False), (128, 128, True), (64, 128, False)])
def test_store_prompts_chunks_and_single_tokens(d, bs, paged, dtype):
    s = Store(3, 2, d, bs, paged, dtype, 3 * bs + 40, seed=d + bs)
    s.store(*s.tokens(bs + 5), new=[bs + 5, 0, bs])       # ragged prompts, one empty
    s.check()
    for _ in range(4):                                    # single tokens
        s.store(*s.tokens(1))
    s.check()
    s.store(*s.tokens(bs + 20), new=[7, bs + 20, bs])     # chunks over block edges
    s.check()
    s.store(*s.tokens(9), new=[0, 9, 1])
    s.check()


def test_store_token_by_token_over_two_blocks():
    s = Store(2, 3, 128, 16, True, "bf16", 40, seed=5)
    for i in range(33):
        s.store(*s.tokens(1, wide=8.0))
    s.check()


def test_store_without_bounds_or_new_lens():
    s = Store(2, 1, 64, 16, False, "f32", 64, seed=6, bounds=False)
    k, v = s.tokens(20)
    s.store(k, v)
    s.check()
    # new_lens NULL: every token; more tokens than the sequence holds: its last ones
    c = s.c
    c.seq.copy_(torch.tensor([20, 12], dtype=I32))
    before = c.dev["k"].view(torch.uint8).clone()
    B.prhs_quant_store(c.kv, k.to(DEV), v.to(DEV))
    after = c.dev["k"].view(torch.uint8)
    assert torch.equal(after[0], before[0])
    want, sc = Q.store_block(np.zeros((0, 64), np.uint8), 1.0, k[1, 0, :12].double().numpy())
    assert np.array_equal(after[1, 0, :12].cpu().numpy(), want) and float(c.dsc["k"][1, 0, 0]) == sc
    assert torch.equal(after[1, 0, 12:], before[1, 0, 12:])


def test_store_extreme_values():
    d, bs = 64, 16
    s = Store(1, 1, d, bs, False, "f32", 7 * bs, seed=7)
    k, v = s.tokens(7 * bs)
    k[0, 0, :16] = 0.0                                         # the smallest scale
    k[0, 0, 16:32] *= 1e-38                                    # denormal numbers
    k[0, 0, 32, 0], k[0, 0, 33, 1] = 3.4e38, -3.4e38           # the largest
    k[0, 0, 48, 0], k[0, 0, 49, 1], k[0, 0, 50, 2] = math.nan, math.inf, -math.inf
    k[0, 0, 64:80] = math.nan                                  # nothing finite
    k[0, 0, 80:96, 0], k[0, 0, 80:96, 1] = 448.0, 480.0        # at the scale's edge
    v[0, 0, :16] = torch.tensor([-0.0])
    # bounds: NaN is left out, and a dimension of nothing but NaN has none
    s.store(k, v)
    s.check()
    s2 = Store(1, 1, d, bs, False, "bf16", bs, seed=8)         # a zero block, then small tokens
    z = torch.zeros(1, 1, 3, d, dtype=torch.bfloat16)
    s2.store(z, z)
    s2.store(*s2.tokens(2, wide=20.0))
    s2.check()


def test_store_drops_tokens_on_pages_outside_the_pool():
    s = Store(2, 2, 128, 16, True, "bf16", 64, seed=9)
    s.c.dtable[0, 1], s.c.dtable[1, 0] = -1, s.c.pages
    s.store(*s.tokens(50), dropped={(0, 1), (1, 0)})
    s.check()


def test_store_is_idempotent():
    s = Store(2, 2, 128, 16, True, "bf16", 64, seed=10)
    s.store(*s.tokens(21))
    k, v = s.tokens(5, wide=6.0)
    s.store(k, v)
    s.check()
    B.prhs_quant_store(s.c.kv, k.to(DEV), v.to(DEV), None, s.bounds)
    s.check()


# ---- bounds and selection ----------------------------------------------------------

def plain_cache(lens, hkv, d, bs, paged, dtype, seed, cap=None):
    """A bf16 or fp32 cache on the grid j/16, NaN behind each sequence."""
    rng = np.random.default_rng(seed)
    n_cap = max(lens) if cap is None else cap
    nb, Bn = -(-n_cap // bs), len(lens)
    x = np.clip(np.round(rng.standard_normal((Bn, hkv, nb * bs, d)) * 16), -255, 255) / 16
    for b, n in enumerate(lens):
        x[b, :, n:] = np.nan
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    seq = torch.tensor(lens, dtype=I32, device=DEV)
    if not paged:
        K = torch.tensor(x, dtype=dt, device=DEV)
        return x, None, seq, K
    pages = Bn * nb + 2
    table = rng.permutation(pages)[: Bn * nb].reshape(Bn, nb)
    phys = np.full((pages, hkv, bs, d), np.nan)
    phys[table.ravel()] = x.reshape(Bn, hkv, nb, bs, d).transpose(0, 2, 1, 3, 4).reshape(-1, hkv, bs, d)
    return x, table, seq, torch.tensor(phys, dtype=dt, device=DEV)


def bounds_of(x, lens, bs, b, g, j):
    return Q.block_bounds(x[b, g, j * bs: min(lens[b], (j + 1) * bs)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,bs,paged", [(128, 16, True), (64, 64, False), (128, 128, False), (64, 32, True)])
def test_block_bounds(d, bs, paged, dtype):
    lens, hkv = (3 * bs + 5, 1, 2 * bs, 0), 2
    x, table, seq, K = plain_cache(lens, hkv, d, bs, paged, dtype, seed=bs + d)
    dtab = torch.tensor(table, dtype=I32, device=DEV) if paged else None
    kv = B.KV(K, K, seq, max(lens), hkv, dtab)
    nb = -(-max(lens) // bs)
    shape = (K.shape[0], hkv, d) if paged else (len(lens), hkv, nb, d)
    for new, cap in (([bs + 7, 1, 1, 0], bs + 9), (None, 1), (None, max(lens) + 50), ([0, 0, 0, 0], 4)):
        lo, hi = (torch.full(shape, v, dtype=K.dtype, device=DEV) for v in (5.0, -5.0))
        nl = None if new is None else torch.tensor(new, dtype=I32, device=DEV)
        B.prhs_block_bounds(kv, B.BlockBounds(kv, lo, hi), cap, nl)
        for b, n in enumerate(lens):
            c = min(n, cap if new is None else min(new[b], cap))
            for g in range(hkv):
                for j in range(nb):
                    at = (int(table[b, j]), g) if paged else (b, g, j)
                    got = lo[at].double().cpu().numpy(), hi[at].double().cpu().numpy()
                    hit = c > 0 and (n - c) // bs <= j and j * bs < n
                    want = bounds_of(x, lens, bs, b, g, j) if hit else (np.full(d, 5.0), np.full(d, -5.0))
                    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1]), (b, g, j, hit)


def run_select(kv, bounds, q, p, bs, max_len, hkv, batch, spare=0):
    kc = max(1, B.prhs_max_blocks(p, bs, max_len)) + spare
    sc = max(1, B.prhs_block_set_capacity(p, bs, max_len)) + spare
    blk, st = (torch.full((batch, hkv, x), -9, dtype=I32, device=DEV) for x in (kc, sc))
    bl, sl = (torch.full((batch, hkv), -9, dtype=I32, device=DEV) for _ in range(2))
    n = B.prhs_block_workspace_size(kv, bounds)
    ws = torch.full((n + 256,), 255, dtype=torch.uint8, device=DEV)
    B.prhs_block_select(kv, q, p, bounds, blk, bl, st, sl, ws[:n])
    assert (ws[n:] == 255).all()
    return blk, bl, st, sl


def check_select(got, sigma, lens, hkv, kb, sink, window, bs):
    blk, bl, st, sl = (t.cpu().numpy() for t in got)
    for b, n in enumerate(lens):
        for g in range(hkv):
            cand = Q.candidate_blocks(n, sink, window, bs)
            want = Q.choose_blocks(sigma(b, g), cand, kb(n), bs)
            S = Q.block_set(want, n, sink, window, bs)
            assert bl[b, g] == len(want) and blk[b, g, : len(want)].tolist() == want, (b, g, n)
            assert sl[b, g] == len(S) and st[b, g, : len(S)].tolist() == S, (b, g, n)
            assert (blk[b, g, len(want):] == -9).all() and (st[b, g, len(S):] == -9).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,bs,paged,n,k,sink,window", [
    (4, 2, 128, 16, True, 700, 96, 4, 32),
    (16, 1, 64, 16, False, 3000, 1000, 0, 0),
    (3, 3, 64, 32, True, 900, 65, 40, 100),        # sink and window end inside blocks
    (5, 1, 128, 64, False, 2000, 1, 16, 64),
    (18, 2, 128, 128, True, 1500, 600, 130, 7),
    (8, 8, 64, 16, False, 400, 5000, 4, 16),       # the budget exceeds the candidates
    (2, 1, 64, 16, True, 300, 0, 4, 16),           # no budget: sink and window
    (2, 1, 64, 16, True, 17000, 512, 4, 64),       # more than a thousand blocks
])
def test_block_select(hq, hkv, d, bs, paged, n, k, sink, window, dtype):
    lens = (n, 0, 1, sink + window, sink + window + 1, n - 1, min(n, sink + bs), 2 * bs)
    lens = tuple(min(x, n) for x in lens)
    x, table, seq, K = plain_cache(lens, hkv, d, bs, paged, dtype, seed=n + k, cap=n)
    dtab = torch.tensor(table, dtype=I32, device=DEV) if paged else None
    kv = B.KV(K, K, seq, n, hq, dtab)
    nb, batch = -(-n // bs), len(lens)
    shape = (K.shape[0], hkv, d) if paged else (batch, hkv, nb, d)
    lo, hi = (torch.full(shape, math.nan, dtype=K.dtype, device=DEV) for _ in range(2))
    bounds = B.BlockBounds(kv, lo, hi)
    B.prhs_block_bounds(kv, bounds, n)
    rng = np.random.default_rng(n)
    q = np.clip(np.round(rng.standard_normal((batch, hq, d)) * 16), -255, 255) / 16
    qd = torch.tensor(q, dtype=K.dtype, device=DEV)
    G = hq // hkv

    def sigma(b, g):
        m = -(-lens[b] // bs)
        if not m:
            return []
        bb = [bounds_of(x, lens, bs, b, g, j) for j in range(m)]
        return Q.block_scores(q[b, g * G:(g + 1) * G], np.array([a for a, _ in bb]), np.array([z for _, z in bb]))

    for p, kb in ((B.params(k=k, sink=sink, window=window), lambda m: k),
                  (B.params(k_num=1, k_den=7, sink=sink, window=window), lambda m: m // 7)):
        got = run_select(kv, bounds, qd, p, bs, n, hkv, batch, spare=3)
        check_select(got, sigma, lens, hkv, kb, sink, window, bs)


@pytest.mark.parametrize("batch,hkv,nb,k,paged,dtype", [
    (1, 2, 8750, 900, True, "bf16"),       # more keys than the picking workgroup's registers hold
    (2, 1, 9000, 80000, False, "f32"),     # more chosen blocks than its LDS holds
    (24, 8, 4300, 3000, False, "bf16"),    # one launch of long rows
    (1, 2, 1500, 640, False, "bf16"), (1, 2, 3000, 900, True, "bf16"), (24, 8, 1500, 640, True, "bf16"),
    (96, 1, 300, 640, True, "bf16"), (96, 1, 600, 640, False, "f32"), (10, 32, 200, 640, False, "bf16"),
])
def test_block_select_long_and_many_rows(batch, hkv, nb, k, paged, dtype):
    bs, d, hq, n = 16, 64, hkv * 2, nb * 16 - 3
    rng = np.random.default_rng(nb)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    lens = tuple(n - (b * 977) % (n // 3) for b in range(batch))
    blocks = batch * nb * hkv
    table = rng.permutation(batch * nb).reshape(batch, nb)
    shape = (batch * nb, hkv, bs, d) if paged else (batch, hkv, nb * bs, d)
    K = torch.empty(shape, dtype=torch.uint8, device=DEV).view(E4)   # not read
    sc = torch.ones(shape[:2] if paged else (batch, hkv, nb), device=DEV)
    kv = B.QuantKV(K, K, sc, sc, torch.tensor(lens, dtype=I32, device=DEV), n, hq,
                   torch.tensor(table, dtype=I32, device=DEV) if paged else None, dtype=dt)
    g = torch.Generator(device=DEV).manual_seed(nb)
    x = torch.randn(blocks, d, generator=g, device=DEV).mul_(16).round_().clamp_(-255, 200).div_(16)
    lo = x.to(dt).view(*sc.shape, d)
    hi = (x + 1.5).to(dt).view(*sc.shape, d)
    q = np.clip(np.round(rng.standard_normal((batch, hq, d)) * 16), -255, 255) / 16
    p = B.params(k=k, sink=20, window=40)
    got = run_select(kv, B.BlockBounds(kv, lo, hi), torch.tensor(q, dtype=dt, device=DEV), p, bs, n, hkv, batch)
    for b in sorted({0, batch // 2, batch - 1}):
        for g_ in sorted({0, hkv - 1}):
            ids = [int(table[b, j]) * hkv + g_ if paged else (b * hkv + g_) * nb + j for j in range(nb)]
            a, z = (t.reshape(-1, d)[ids].double().cpu().numpy() for t in (lo, hi))
            sig = Q.block_scores(q[b, 2 * g_:2 * g_ + 2], a, z)
            check_select([t[b:b + 1, g_:g_ + 1] for t in got], lambda *_: sig, [lens[b]], 1, lambda m: k, 20, 40, bs)


@pytest.mark.parametrize("paged", [False, True])
def test_block_select_ties_nan_and_lost_pages(paged):
    # equal scores everywhere: the lowest blocks; a block of NaN bounds and one on
    # a page outside the pool rank last
    n, bs, d, hkv = 2000, 16, 64, 2
    nb = -(-n // bs)
    lens = (n, n - 5)
    table = np.arange(2 * nb).reshape(2, nb)
    K = torch.zeros((2 * nb, hkv, bs, d) if paged else (2, hkv, nb * bs, d), dtype=torch.bfloat16, device=DEV)
    dtab = torch.tensor(table, dtype=I32, device=DEV) if paged else None
    kv = B.KV(K, K, torch.tensor(lens, dtype=I32, device=DEV), n, 4, dtab)
    lo = torch.zeros((2 * nb, hkv, d) if paged else (2, hkv, nb, d), dtype=torch.bfloat16, device=DEV)
    hi = lo.clone()
    at = lambda b, g, j: (int(table[b, j]), g) if paged else (b, g, j)  # noqa: E731
    sig = {(b, g): np.zeros(nb) for b in range(2) for g in range(hkv)}
    for g in range(hkv):
        hi[at(0, g, 3)][0] = math.nan
        sig[0, g][3] = -math.inf
        hi[at(1, g, 60)][5] = 2.0
        sig[1, g][60] = 2.0
        lo[at(1, g, 61)].fill_(-0.0)
    if paged:
        dtab[1, 5] = 2 * nb
        for g in range(hkv):
            sig[1, g][5] = -math.inf
    q = torch.ones(2, 4, d, dtype=torch.bfloat16, device=DEV)
    for k in (16, 160, 1600, 4000):
        p = B.params(k=k, sink=0, window=0)
        got = run_select(kv, B.BlockBounds(kv, lo, hi), q, p, bs, n, hkv, 2)
        check_select(got, lambda b, g: sig[b, g], lens, hkv, lambda m: k, 0, 0, bs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_block_select_infinite_bounds(dtype):
    # a score of +inf ranks first, ties to the lower block; where an infinite bound
    # meets a zero of q's positive or negative part the score is NaN and ranks last
    n, bs, d, hkv = 700, 32, 128, 2
    nb = -(-n // bs)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    K = torch.zeros((1, hkv, nb * bs, d), dtype=dt, device=DEV)
    kv = B.KV(K, K, torch.tensor([n], dtype=I32, device=DEV), n, 4)
    lo = torch.zeros((1, hkv, nb, d), dtype=dt, device=DEV)
    hi = lo.clone()
    hi[:, :, 3, 0] = math.inf    # q > 0
    lo[:, :, 7, 0] = -math.inf
    hi[:, :, 9, 1] = math.inf    # q < 0
    lo[:, :, 11, 1] = -math.inf
    sig = np.zeros(nb)
    sig[[3, 11]], sig[[7, 9]] = math.inf, -math.inf
    q = torch.ones(1, 4, d, dtype=dt, device=DEV)
    q[:, :, 1] = -1.0
    for k in (32, 64, 96, bs * (nb - 2), bs * (nb - 1)):
        got = run_select(kv, B.BlockBounds(kv, lo, hi), q, B.params(k=k, sink=0, window=0), bs, n, hkv, 1)
        check_select(got, lambda b, g: sig, (n,), hkv, lambda m: k, 0, 0, bs)


# ---- together ----------------------------------------------------------------------

def test_store_select_and_attend_as_a_decode_loop():
    """A prompt and seven steps: store, a selection of blocks every third step,
    attention over the set and the tokens since."""
    batch, hq, hkv, d, bs, T, P = 2, 8, 2, 128, 16, 7, 150
    s = Store(batch, hkv, d, bs, True, "bf16", P + T, seed=20)
    c = s.c
    c.hq = hq
    kv = B.QuantKV(c.dev["k"], c.dev["v"], c.dsc["k"], c.dsc["v"], c.seq, P + T, hq, c.dtable)
    c.kv = kv
    grid = lambda x: (x.float() * 16).round().clamp(-255, 255).div(16).to(x.dtype)  # noqa: E731
    s.bounds = B.BlockBounds(kv, s.dlo, s.dhi)
    k, v = s.tokens(P, wide=1.0)
    s.store(grid(k), v, new=[P, P - 37])
    p = B.params(k=48, sink=4, window=20, refresh_every=3)
    got = None
    for j in range(T):
        k, v = s.tokens(1, wide=1.0)
        s.store(grid(k), v)
        s.check()
        q = grid(torch.tensor(np.random.default_rng(j).standard_normal((batch, hq, d)), dtype=torch.bfloat16))
        c.q, c.lens = q.to(DEV), tuple(s.n)
        if j % 3 == 0:
            got = run_select(kv, s.bounds, c.q, p, bs, P + T, hkv, batch)
            anchor, sets = c.seq.clone(), {}
            for b, n in enumerate(s.n):
                for g in range(hkv):
                    ids = [c.block(b, g, i) for i in range(-(-n // bs))]
                    sig = Q.block_scores(q[b, g * 4:(g + 1) * 4].double().numpy(), s.lo[ids], s.hi[ids])
                    blocks = Q.choose_blocks(sig, Q.candidate_blocks(n, 4, 20, bs), 48, bs)
                    sets[b, g] = Q.block_set(blocks, n, 4, 20, bs)
                    assert got[2][b, g, : len(sets[b, g])].tolist() == sets[b, g]
        y, lse = c.outputs()
        cap = got[2].shape[2]
        B.prhs_quant_reuse_decode_attn(kv, c.q, got[2], got[3], anchor, c.scale_q, y, lse, c.workspace(False, cap))
        n0 = anchor.tolist()
        c.check(y, lse, lambda b, g: sets[b, g] + list(range(n0[b], s.n[b])))


@pytest.mark.parametrize("paged", [True, False])
def test_bytes_behind_four_gigabytes(paged):
    # the last pages, or the last unit's rows, of a cache that lie behind 2^32 bytes
    # give what a small cache gives, and nothing else is written
    batch, hq, hkv, d, bs, n = 2, 8, 4, 128, 64, 700
    nb = -(-n // bs)
    big = 2 ** 32 // ((hkv if paged else batch * hkv - 1) * bs * d) + (batch * nb if paged else 1)
    g = torch.Generator(device=DEV).manual_seed(9)
    k, v = (torch.randn(batch, hkv, n, d, generator=g, device=DEV).bfloat16() for _ in "kv")
    q = torch.randn(batch, hq, d, generator=g, device=DEV).bfloat16()
    seq = torch.tensor([n, n - 70], dtype=I32, device=DEV)
    p = B.params(k=200, sink=4, window=30)
    got = []
    for blocks in (batch * nb, big) if paged else (nb, big):
        lead = (blocks, hkv) if paged else (batch, hkv, blocks)
        shape = (blocks, hkv, bs, d) if paged else (batch, hkv, blocks * bs, d)
        K, V = (torch.zeros(shape, dtype=torch.uint8, device=DEV) for _ in "kv")
        ks, vs = (torch.ones(lead, device=DEV) for _ in "kv")
        table = None
        if paged:
            table = (blocks - 1 - torch.arange(batch * nb, device=DEV)).view(batch, nb).to(I32)
        kv = B.QuantKV(K.view(E4), V.view(E4), ks, vs, seq, n, hq, table)
        lo, hi = (torch.zeros(*lead, d, dtype=torch.bfloat16, device=DEV) for _ in "kv")
        bounds = B.BlockBounds(kv, lo, hi)
        B.prhs_quant_store(kv, k, v, None, bounds)
        sel = run_select(kv, bounds, q, p, bs, n, hkv, batch)
        outs = []
        for op in (B.PRHS_OP_QUANT_DENSE_ATTN, B.PRHS_OP_QUANT_SPARSE_ATTN):
            y, lse = torch.zeros(batch, hq, d, device=DEV), torch.zeros(batch, hq, device=DEV)
            ws = B.workspace(B.prhs_workspace_size(op, kv, None, sel[2].shape[2]), DEV)
            if op == B.PRHS_OP_QUANT_DENSE_ATTN:
                B.prhs_quant_dense_decode_attn(kv, q, 0.1, y, lse, ws)
            else:
                B.prhs_quant_sparse_decode_attn(kv, q, sel[2], sel[3], 0.1, y, lse, ws)
            outs += [y, lse]
        used = table.flatten().long() if paged else None
        rows = [x[used] if paged else x[:, :, : nb * bs] for x in (K, V)]
        outs += [*rows, *(x[used] if paged else x[:, :, :nb] for x in (ks, vs, lo, hi)), *sel]
        outs += [sum(int(t.count_nonzero()) for t in x.view(-1).split(2 ** 28)) for x in (K, V)]
        got.append(outs)
    for i, (a, b) in enumerate(zip(*got)):
        assert a == b if isinstance(a, int) else torch.equal(a, b), i


def test_graph_replays_equal_the_eager_calls():
    batch, hq, hkv, d, bs, n = 3, 8, 2, 64, 16, 3000
    lens = (n, 1200, 65)
    c = Cache(lens, hq, hkv, d, bs, True, "bf16", seed=30)
    lo = torch.randn(c.pages, hkv, d, device=DEV).bfloat16()
    bounds = B.BlockBounds(c.kv, lo, lo + 1)
    p = B.params(k=256, sink=4, window=32)
    kc, sc = B.prhs_max_blocks(p, bs, n), B.prhs_block_set_capacity(p, bs, n)
    blk, st = (torch.zeros(batch, hkv, x, dtype=I32, device=DEV) for x in (kc, sc))
    bl, sl = (torch.zeros(batch, hkv, dtype=I32, device=DEV) for _ in range(2))
    wb = B.workspace(B.prhs_block_workspace_size(c.kv, bounds), DEV)
    ws = B.workspace(max(B.prhs_workspace_size(B.PRHS_OP_QUANT_SPARSE_ATTN, c.kv, None, sc),
                         B.prhs_workspace_size(B.PRHS_OP_QUANT_DENSE_ATTN, c.kv)), DEV)
    k1, v1 = (torch.randn(batch, hkv, 1, d, device=DEV).bfloat16() for _ in "kv")
    y, lse = c.outputs()
    z, zse = c.outputs()

    def step():
        B.prhs_quant_store(c.kv, k1, v1, None, bounds)
        B.prhs_block_select(c.kv, c.q, p, bounds, blk, bl, st, sl, wb)
        B.prhs_quant_sparse_decode_attn(c.kv, c.q, st, sl, c.scale_q, y, lse, ws)
        B.prhs_quant_dense_decode_attn(c.kv, c.q, c.scale_q, z, zse, ws)

    state = [*c.dev.values(), *c.dsc.values(), lo, bounds._keep[1], blk, bl, st, sl, y, lse, z, zse]
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in state]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        for t in (blk, bl, st, sl, y, lse, z, zse):
            t.zero_()
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(state, want):
            va, vb = (t.view(torch.uint8) if t.dtype == E4 else t for t in (a, b))
            assert torch.equal(torch.nan_to_num(va.float()), torch.nan_to_num(vb.float()))
        torch.randn(1000, device=DEV).sum().item()   # eager work between the replays


def every_call(monkeypatch=None):
    """Outputs of one call of every entry point of the 8-bit cache and the blocks."""
    res = []

    def keep(*shape, dtype=I32):
        res.append(torch.zeros(*shape, dtype=dtype, device=DEV))
        return res[-1]

    lens, hq, hkv, d = (300, 77), 8, 2, 64
    c = Cache(lens, hq, hkv, d, 16, True, "bf16", seed=40)
    lo = torch.randn(c.pages, hkv, d, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).bfloat16()
    hi = lo + 1
    bounds = B.BlockBounds(c.kv, lo, hi)
    new = torch.ones(2, hkv, 3, d, dtype=torch.bfloat16, device=DEV)
    B.prhs_quant_store(c.kv, new, new, torch.tensor([2, 3], dtype=I32, device=DEV), bounds)
    B.prhs_quant_store(c.kv, new, new)
    p = B.params(k=40, sink=4, window=8)
    kc, sc = B.prhs_max_blocks(p, 16, 300), B.prhs_block_set_capacity(p, 16, 300)
    blk, bl, st, sl = keep(2, hkv, kc), keep(2, hkv), keep(2, hkv, sc), keep(2, hkv)
    B.prhs_block_select(c.kv, c.q, p, bounds, blk, bl, st, sl, B.workspace(B.prhs_block_workspace_size(c.kv, bounds), DEV))
    ws = B.workspace(max(B.prhs_workspace_size(B.PRHS_OP_QUANT_SPARSE_ATTN, c.kv, None, sc),
                         B.prhs_workspace_size(B.PRHS_OP_QUANT_DENSE_ATTN, c.kv)), DEV)
    f32 = dict(dtype=torch.float32)
    ids, tail = torch.arange(4, dtype=I32, device=DEV), c.seq.repeat_interleave(2).contiguous()
    out = lambda: (keep(2, hq, d, **f32), keep(2, hq, **f32))  # noqa: E731
    B.prhs_quant_dense_decode_attn(c.kv, c.q, c.scale_q, *out(), ws)
    B.prhs_quant_sparse_decode_attn(c.kv, c.q, st, sl, c.scale_q, *out(), ws)
    B.prhs_quant_reuse_decode_attn(c.kv, c.q, st, sl, c.seq, c.scale_q, *out(), ws)
    B.prhs_quant_pool_decode_attn(c.kv, c.q, st, sl, ids, tail, c.scale_q, *out(), ws, psaw=B.psaw(3, 4, 1, 0.5, 1.0, 4))
    K = torch.randn(2, hkv, 320, d, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).bfloat16()
    kv = B.KV(K, K, c.seq, 300, hq)
    bb = B.BlockBounds(kv, keep(2, hkv, 20, d, dtype=torch.bfloat16), keep(2, hkv, 20, d, dtype=torch.bfloat16))
    B.prhs_block_bounds(kv, bb, 300)
    B.prhs_block_select(kv, c.q, p, bb, keep(2, hkv, kc), keep(2, hkv), keep(2, hkv, sc), keep(2, hkv),
                        B.workspace(B.prhs_block_workspace_size(kv, bb), DEV))
    torch.cuda.synchronize()
    return res + [c.dev["k"].view(torch.uint8), c.dev["v"].view(torch.uint8), lo, hi]


def test_native_marshalling_equals_python(monkeypatch):
    if B._host is None:
        pytest.skip("the extension is not built")
    host, taken = B._host, []

    class Watch:
        def __getattr__(self, name):
            def f(*a):
                r = getattr(host, name)(*a)
                if r is not None:
                    taken.append(name)
                return r
            return f

    monkeypatch.setattr(B, "_host", Watch())
    native = every_call()
    assert set(taken) == {"quant_store", "quant_dense", "quant_sparse", "quant_reuse", "quant_pool", "block_bounds", "block_select"}
    assert taken.count("block_select") == 2 and taken.count("quant_store") == 2
    monkeypatch.setattr(B, "_host", None)
    for x, y in zip(native, every_call()):
        assert torch.equal(x, y)


def test_what_does_not_fit_raises_from_the_native_path_too():
    c = Cache((300, 77), 8, 2, 64, 16, True, "bf16", seed=41)
    y, lse = c.outputs()
    ws = c.workspace(True)
    new = torch.ones(2, 2, 3, 64, dtype=torch.bfloat16, device=DEV)
    for bad in (lambda: B.prhs_quant_dense_decode_attn(c.kv, c.q.float(), 1.0, y, lse, ws),
                lambda: B.prhs_quant_dense_decode_attn(c.kv, c.q.cpu(), 1.0, y, lse, ws),
                lambda: B.prhs_quant_dense_decode_attn(c.kv, c.q, 1.0, y[:1], lse, ws),
                lambda: B.prhs_quant_store(c.kv, new, new[:, :1].contiguous()),
                lambda: B.prhs_quant_store(c.kv, new, new, torch.zeros(3, dtype=I32, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.PrhsError) as e:
        B.prhs_quant_dense_decode_attn(c.kv, c.q, 1.0, y, lse, ws[:16])
    assert e.value.status == B.PRHS_E_WORKSPACE
    assert (y == 7).all()
