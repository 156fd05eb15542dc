"""The decode schedule over an 8-bit cache (QuantDecodeRunner): every step's
sets are those of the oracle on the cache's own bounds, the outputs the
attention of the values that the cache stands for, and graph replays equal the
eager steps."""

import math

import numpy as np
import pytest
import torch

import oracle as O
from oracle import quant_oracle as Q
from paper_2602_08329_amd import binding as B
from paper_2602_08329_amd import synth
from paper_2602_08329_amd.schedule import QuantDecodeRunner, capture_steps
from tests.quant_tolerance import assert_attention

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def workload(index, **kw):
    w = synth.workload(index)
    return w.replace(**kw)


CASES = [
    (workload(0, steps=9), 32),                                                       # fp32, MHA
    (workload(2, layers=6, n_ctx=(700, 300), batch=2, k=100, window=40, steps=10, s=4, G=4), 16),
    (workload(3, layers=2, n_ctx=(1500,), k=200, window=64, steps=6, s=3), None),     # paged
]


class Stored:
    """A layer's cache, read back: blocks, scales and bounds of a unit."""

    def __init__(self, run, l):
        kv = run.kv[l][0]
        K8, V8, ks, vs, _, table = kv._keep
        self.paged, self.bs = table is not None, run.block_size
        self.t = None if table is None else table.cpu().numpy()
        self.raw = [x.view(torch.uint8).cpu().numpy() for x in (K8, V8)]
        self.sc = [x.double().cpu().numpy() for x in (ks, vs)]
        self.bd = [x.double().cpu().numpy() for x in run.bounds[l]._keep]

    def blocks(self, x, b, g, n):
        m = -(-n // self.bs)
        return x[self.t[b, :m], g] if self.paged else x[b, g, :m]

    def values(self, i, b, g, n):
        m = -(-n // self.bs)
        r = self.blocks(self.raw[i], b, g, n) if self.paged else self.raw[i][b, g, : m * self.bs].reshape(m, self.bs, -1)
        return (Q.TABLE[r] * self.blocks(self.sc[i], b, g, n)[:, None, None]).reshape(m * self.bs, -1)[:n]


@pytest.mark.parametrize("w,block", CASES)
def test_steps_match_the_oracle(w, block):
    inp = synth.generate(w, device=DEV)
    run = QuantDecodeRunner(inp, block_size=block or 16)
    g = w.hq // w.hkv
    units = [(0, 0), (w.batch - 1, w.hkv - 1)]
    sets = {}
    for j in range(w.steps):
        outs = [(torch.full_like(run.out, 7.0), torch.full_like(run.lse, 7.0)) for _ in range(run.L)]
        run.step(j, outs)
        kb = lambda n: O.budget_k(n, k=w.k if not w.k_den else None, k_num=w.k_num, k_den=w.k_den)  # noqa: E731
        for l in range(run.L):
            st, gi = Stored(run, l), l // w.G
            for b, hk in units:
                n = w.n_ctx[b] + j + 1
                q = inp.q[l, j, b, hk * g:(hk + 1) * g].double().cpu().numpy()
                if l % w.G == 0 and j % w.s == 0:
                    lo, hi = (st.blocks(x, b, hk, n) for x in st.bd)
                    sig = Q.block_scores(q, lo, hi)
                    blocks = Q.choose_blocks(sig, Q.candidate_blocks(n, w.sink, w.window, st.bs), kb(n), st.bs)
                    sets[gi, b, hk] = (n, Q.block_set(blocks, n, w.sink, w.window, st.bs))
                n0, S = sets[gi, b, hk]
                got = run.sets[gi][0][b, hk, : int(run.sets[gi][1][b, hk])].tolist()
                assert got == S
                K, V = (st.values(i, b, hk, n)[S + list(range(n0, n))] for i in (0, 1))
                for h in range(g):
                    yr, lr = O.dense_attention(q[h], K, V)
                    y = outs[l][0][b, hk * g + h].double().cpu().numpy()
                    assert_attention(y, float(outs[l][1][b, hk * g + h]), yr, lr, q[h], K, V,
                                     1 / math.sqrt(w.d), (j, l, b, hk, h))
    # the cache holds the tokens within its precision: half a step of the block's
    # scale, 2^-4 relative or 2^-10 of it
    for b, hk in units:
        n = w.n_ctx[b] + w.steps
        for i, X in enumerate((inp.K[0], inp.V[0])):
            want = run._in_order(X, run.kv[0][0]._keep[5])[b, hk, :n].double().cpu().numpy()
            st = Stored(run, 0)
            s = np.repeat(st.blocks(st.sc[i], b, hk, n), st.bs)[:n, None]
            # elements stored before their block's scale grew are rounded once more
            tol = np.maximum(np.abs(want) * 2.0 ** -4, s * 2.0 ** -10) + s * 2.0 ** -10
            assert (np.abs(st.values(i, b, hk, n) - want) <= tol).all()


def test_graph_replays_equal_the_eager_steps():
    w = CASES[1][0]
    inp = synth.generate(w, device=DEV)
    run, ref = QuantDecodeRunner(inp), QuantDecodeRunner(inp)
    bufs = {(l, j): (torch.empty_like(run.out), torch.empty_like(run.lse)) for l in range(run.L) for j in range(w.steps)}
    want = {k: (torch.empty_like(run.out), torch.empty_like(run.lse)) for k in bufs}
    for j in range(w.steps):
        ref.step(j, [want[l, j] for l in range(run.L)])
    run.step(0)
    graph = capture_steps(lambda j: run.step(j, [bufs[l, j] for l in range(run.L)]), range(w.steps))
    fresh = [t.clone() for t in first_state(run)]
    for _ in range(3):
        for t, f in zip(first_state(run), fresh):   # the caches as before the steps
            t.copy_(f)
        for y, s in bufs.values():
            y.fill_(math.nan)
            s.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        for k in bufs:
            assert torch.equal(bufs[k][0], want[k][0]) and torch.equal(bufs[k][1], want[k][1]), k
        torch.randn(1000, device=DEV).sum().item()


def first_state(run):
    return [t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
            for l in range(run.L) for t in (*run.kv[l][0]._keep[:4], *run.bounds[l]._keep)]


def test_steps_out_of_order_are_refused():
    inp = synth.generate(CASES[1][0], device=DEV, layers=1)
    run = QuantDecodeRunner(inp)
    with pytest.raises(RuntimeError, match="no anchor"):
        run.attend(0, 0)
    run.step(0)
    with pytest.raises(RuntimeError, match="no anchor"):
        run.attend(0, 4)
