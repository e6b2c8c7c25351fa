"""Attention over packed sequences, shared prefixes, and the norms of queries and keys with the rotation, on the GPU, against plain float64
implementations on the CPU, through the C ABI.

Tolerances are counted in roundings u = half a step relative to the value (bf16 2^-8 ... `finfo.eps / 2`; fp32 2^-24):
  bf16  an output is rounded once (u / sqrt(3) of its size in the 2-norm on average, at most u), the probabilities (or score gradients)
        that make it once before their product (the same, independent), and delta inherits O's rounding: relative 2-norm error below
        sqrt(1 + 1 + 1) u / sqrt(3) = u; held to 1.5 u = 6e-3.  Elements: 8 of those, relative to the larger of the element and the row's rms.
  fp32  sums of n products in any order: below sqrt(n) u on average, exp2 / log2 within 2 u of arguments up to 2^5 units (error 2^5 u on
        an exponent): 2-norm below (sqrt(n) + 64) u, n at most 4096: 128 u = 8e-6; held to 1e-5.
Gradients of queries and keys cancel: dS = P (dP - delta) can be far smaller than P |dP| and P |delta|, and an element of dK = sum dS q far smaller
than its terms, so no factor on the element or on the rms bounds its error.  Their elements are held to the sum of what can happen to
each term instead (`bounds` of the oracle), which for dK[u] is, with v = u of the storage type and c = 1e-5 for the fp32 arithmetic,
  sum_i scale |q_i| (v |dS_iu| + P_iu v sum_d |dO_id O_id| + c P_iu (sum_d |dO_id V_ud| + sum_d |dO_id O_id|)) + v |dK|
(dS rounded before its product; delta computed from the rounded O; the result rounded), and likewise for dQ with keys for queries.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2312_07987_amd import binding

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
REL = {"f32": 1e-5, "bf16": 6e-3}
NEG = -math.inf


def close(name, got, ref, dtype, scale=None):
    got, ref = got.double().cpu(), ref.double()
    assert got.shape == ref.shape, name
    fin = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), fin) and torch.equal(got[~fin], ref[~fin]), name
    got, ref = got[fin], ref[fin]
    if ref.numel() == 0:
        return
    norm = float(ref.norm()) if scale is None else scale
    err = float((got - ref).norm())
    print(name, "rel %.2e" % (err / norm if norm else err), flush=True)
    assert err <= REL[dtype] * norm + 1e-30, (name, err, norm)
    rms = norm / math.sqrt(ref.numel())
    worst = float(((got - ref).abs() / torch.clamp(ref.abs(), min=max(rms, 1e-30))).max())
    assert worst <= 8 * REL[dtype], (name, worst)


def oracle(q, k, v, nq, nk, group, causal, scale, kp=None, vp=None, dO=None, unit=0.0):
    """One sequence in float64: q [nq, H, d], k, v [nk, Hk, d].  A hidden key takes no part, whatever it holds.  grads[3], grads[4]: how far
    elements of dQ and dK may be off, with roundings of `unit`."""
    H, d = q.shape[1], q.shape[2]
    O, lse = torch.zeros(nq, H, d, dtype=torch.float64), torch.full((H, nq), NEG, dtype=torch.float64)
    grads = [torch.zeros(t, dtype=torch.float64) for t in (q.shape, k.shape, k.shape, q.shape, k.shape)]
    vis = torch.ones(nq, nk, dtype=torch.bool)
    if causal:
        vis = torch.arange(nk)[None] <= (nk - nq) + torch.arange(nq)[:, None]
    for h in range(H):
        kk, vv, see = k[:, h // group], v[:, h // group], vis
        if kp is not None:
            kk, vv = torch.cat((kp[:, h // group], kk)), torch.cat((vp[:, h // group], vv))
            see = torch.cat((torch.ones(nq, kp.shape[0], dtype=torch.bool), vis), 1)
        for i in range(nq):
            at = see[i].nonzero()[:, 0]
            if at.numel() == 0:
                continue
            s = kk[at] @ q[i, h] * scale
            lse[h, i] = torch.logsumexp(s, 0)
            p = torch.exp(s - lse[h, i])
            O[i, h] = p @ vv[at]
            if dO is not None:
                dp = vv[at] @ dO[i, h]
                ds = p * (dp - (p * dp).sum()) * scale
                grads[0][i, h] = ds @ kk[at]
                grads[1][at, h // group] += ds[:, None] * q[i, h]
                grads[2][at, h // group] += p[:, None] * dO[i, h]
                terms = (dO[i, h] * O[i, h]).abs().sum()
                off = unit * ds.abs() + p * scale * (unit * terms + 1e-5 * (vv[at].abs() @ dO[i, h].abs() + terms))
                grads[3][i, h] = off @ kk[at].abs()
                grads[4][at, h // group] += off[:, None] * q[i, h].abs()
    grads[3] += unit * grads[0].abs()
    grads[4] += unit * grads[1].abs()
    return O, lse, grads


class Packed:
    """Host tensors of packed sequences, already rounded to the storage type, and their places."""

    def __init__(self, H, Hk, d, dtype, nq, nk=None, causal=1, prefix=0, seed=0, gap=0, fused=False, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        nk = list(nq) if nk is None else nk
        self.H, self.Hk, self.d, self.dtype, self.nq, self.nk, self.causal, self.prefix = H, Hk, d, dtype, list(nq), list(nk), causal, prefix
        # gap > 0: every sequence's place is that much longer than its length, and rows lie in front of the first
        self.qoff, self.koff = [gap], [gap]
        for a, b in zip(nq, nk):
            self.qoff.append(self.qoff[-1] + a + gap)
            self.koff.append(self.koff[-1] + b + gap)
        self.gap = gap
        Nq, Nk = self.qoff[-1] + gap, self.koff[-1] + gap
        if fused:
            assert self.nq == self.nk
        rnd = lambda *s: (torch.randn(*s, generator=g) * spread).to(DT[dtype])
        if fused:
            t = rnd(max(Nq, 1), H + 2 * Hk, d)
            self.q, self.k, self.v = t[:, :H], t[:, H:H + Hk], t[:, H + Hk:]
            self.fused = t
        else:
            self.q, self.k, self.v = rnd(Nq, H, d), rnd(Nk, Hk, d), rnd(Nk, Hk, d)
            self.fused = None
        self.dO = rnd(Nq, H, d)
        self.kp, self.vp = (rnd(prefix, Hk, d), rnd(prefix, Hk, d)) if prefix else (None, None)
        self.scale = 1.0 / math.sqrt(d)

    def device(self):
        if self.fused is not None:
            t = self.fused.cuda()
            return t[:, :self.H], t[:, self.H:self.H + self.Hk], t[:, self.H + self.Hk:]
        return self.q.cuda(), self.k.cuda(), self.v.cuda()

    def run(self, backward=False, max_q=None, max_k=None, fill=777.0, scale=0.0, lse_wanted=True, ws_fill=None):
        q, k, v = self.device()
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        qoff, koff = i32(self.qoff), i32(self.koff)
        qlen, klen = (i32(self.nq), i32(self.nk)) if self.gap else (None, None)
        O = torch.full(self.q.shape, fill, dtype=q.dtype, device="cuda")
        lse = torch.full((self.H, self.q.shape[0]), fill, device="cuda") if lse_wanted else None
        kp, vp = (self.kp.cuda(), self.vp.cuda()) if self.prefix else (None, None)
        plan = binding.make_attention(q, k, v, O, len(self.nq), max(self.nq) if max_q is None else max_q, max(self.nk) if max_k is None else max_k,
                                      self.causal, kp, vp, scale)
        nbytes = max(binding.switchhead_attention_workspace_bytes(plan), binding.switchhead_attention_workspace_bytes(plan, True) if backward else 0)
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        ws.fill_(255 if ws_fill is None else ws_fill)   # NaN everywhere
        binding.switchhead_attention_forward(plan, q, k, v, qoff, koff, O, lse, ws, qlen, klen, kp, vp)
        out = dict(O=O, lse=lse)
        if backward:
            ws.fill_(255)
            if self.fused is not None:
                t = torch.full(self.fused.shape, fill, dtype=q.dtype, device="cuda")
                dq, dk, dv = t[:, :self.H], t[:, self.H:self.H + self.Hk], t[:, self.H + self.Hk:]
            else:
                dq, dk, dv = (torch.full(x.shape, fill, dtype=q.dtype, device="cuda") for x in (q, k, v))
            binding.switchhead_attention_backward(plan, q, k, v, O, self.dO.cuda(), lse, qoff, koff, dq, dk, dv, ws, qlen, klen)
            out.update(dQ=dq, dK=dk, dV=dv)
        torch.cuda.synchronize()
        return out

    def reference(self, backward=False, fill=777.0):
        w = lambda t: t.double()
        O, lse = torch.full(self.q.shape, fill, dtype=torch.float64), torch.full((self.H, self.q.shape[0]), fill, dtype=torch.float64)
        gr = [torch.full(t.shape, fill, dtype=torch.float64) for t in (self.q, self.k, self.v, self.q, self.k)]
        kp, vp = (w(self.kp), w(self.vp)) if self.prefix else (None, None)
        for i, (a, b) in enumerate(zip(self.nq, self.nk)):
            qs, ks = slice(self.qoff[i], self.qoff[i] + a), slice(self.koff[i], self.koff[i] + b)
            o, l, g = oracle(w(self.q[qs]), w(self.k[ks]), w(self.v[ks]), a, b, self.H // self.Hk, self.causal, self.scale, kp, vp,
                             w(self.dO[qs]) if backward else None, torch.finfo(DT[self.dtype]).eps / 2)
            O[qs], lse[:, qs] = o, l
            gr[0][qs], gr[1][ks], gr[2][ks], gr[3][qs], gr[4][ks] = g
        out = dict(O=O, lse=lse)
        if backward:
            out.update(dQ=gr[0], dK=gr[1], dV=gr[2], bounds=dict(dQ=gr[3], dK=gr[4]))
        return out

    def check(self, backward=False, **kw):
        got, ref = self.run(backward, **kw), self.reference(backward)
        bounds = ref.pop("bounds", {})
        # the rows of sequences together, and the others exactly as they were
        mine = {"q": torch.zeros(self.q.shape[0], dtype=torch.bool), "k": torch.zeros(self.k.shape[0], dtype=torch.bool)}
        for i, (a, b) in enumerate(zip(self.nq, self.nk)):
            mine["q"][self.qoff[i]:self.qoff[i] + a] = True
            mine["k"][self.koff[i]:self.koff[i] + b] = True
        for name in ref:
            if got[name] is None:
                continue
            x, y = got[name].double().cpu(), ref[name]
            m = mine["k" if name in ("dK", "dV") else "q"]
            if name == "lse":
                x, y = x.t(), y.t()
            assert torch.equal(x[~m], y[~m].to(got[name].dtype).double()), name
            x, y = x[m], y[m]
            if name in bounds:
                over = (x - y).abs() - bounds[name][m]
                print(name, "most of its bound %.2f" % float(((x - y).abs() / (bounds[name][m] + 1e-30)).max()) if y.numel() else "")
                assert y.numel() == 0 or float(over.max()) <= 0, (name, float(over.max()))
            else:
                close(name, x, y, "f32" if name == "lse" else self.dtype)
        return got


SHAPES = [   # H, Hk, d
    (2, 2, 32), (4, 4, 128), (8, 2, 64), (5, 1, 80), (2, 2, 76), (3, 3, 41), (6, 2, 100), (2, 1, 256), (2, 2, 8), (1, 1, 1), (4, 2, 132),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d", SHAPES)
def test_ragged_training_batches(H, Hk, d, dtype):
    """Lengths of one token to past a tile, empty sequences between them, forward and gradients."""
    Packed(H, Hk, d, dtype, [1, 0, 33, 130, 2, 0, 64, 65], seed=d).check(backward=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d", [(4, 1, 128), (2, 2, 64), (2, 2, 76), (2, 1, 256)])
def test_more_keys_than_queries_and_fewer(H, Hk, d, dtype):
    """Queries behind keys that are there already; queries that come before every key see nothing: zeros, -inf and no gradient."""
    Packed(H, Hk, d, dtype, [5, 70, 40, 3, 20, 7], [133, 70, 300, 0, 7, 64], seed=3).check(backward=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d", [(2, 2, 64), (8, 2, 128)])
def test_without_causal_mask(H, Hk, d, dtype):
    Packed(H, Hk, d, dtype, [5, 70, 1, 129], [33, 70, 200, 64], causal=0, seed=4).check(backward=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d", [(4, 4, 128), (6, 2, 76), (2, 2, 41)])
def test_views_of_a_fused_projection(H, Hk, d, dtype):
    Packed(H, Hk, d, dtype, [40, 129, 7], fused=True, seed=5).check(backward=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("queries", [[1, 1, 1, 1], [90, 3, 0, 64]])
def test_padded_batch_leaves_other_rows(dtype, queries):
    """Places longer than the sequences: rows behind them keep what they held, and what K and V hold there has no influence."""
    p = Packed(4, 2, 64, dtype, queries, [90, 3, 200, 64], gap=37, seed=6)
    for i, n in enumerate(p.nk):
        for t in (p.k, p.v):
            t[p.koff[i] + n:p.koff[i + 1]] = float("nan")
    p.k[:p.gap], p.v[:p.gap] = float("inf"), float("nan")
    for i, n in enumerate(p.nq):
        p.q[p.qoff[i] + n:p.qoff[i + 1]] = float("nan")
        p.dO[p.qoff[i] + n:p.qoff[i + 1]] = float("nan")
    p.check(backward=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d", [(4, 4, 128), (8, 1, 64), (5, 1, 80), (2, 2, 76), (3, 3, 41), (4, 2, 256), (1, 1, 1)])
@pytest.mark.parametrize("keys", [[1, 700, 33, 64], [3000, 5, 1, 129]])
def test_single_tokens_over_caches(H, Hk, d, dtype, keys):
    Packed(H, Hk, d, dtype, [1] * len(keys), keys, seed=7).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_few_tokens_over_caches(dtype):
    Packed(4, 2, 128, dtype, [3, 8, 0, 1, 5], [3, 600, 20, 0, 2], seed=8).check()
    Packed(4, 2, 128, dtype, [3, 8, 0, 1, 5], [3, 600, 20, 0, 2], seed=8, gap=100).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_cache_of_one_sequence_splits(dtype):
    Packed(4, 1, 64, dtype, [2], [5001], seed=9).check()
    Packed(2, 2, 128, dtype, [40], [3001], seed=10).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("queries,keys", [([1] * 9, [1, 5, 0, 64, 65, 2, 300, 1, 7]), ([20, 1, 7, 90], [20, 1, 9, 90]), ([200, 150], [200, 300]),
                                          ([3, 0, 5], [0, 0, 2]), ([30] * 5, [30, 10, 0, 64, 31])])
@pytest.mark.parametrize("prefix", [1, 64, 333])
def test_shared_prefix(dtype, queries, keys, prefix):
    Packed(4, 2, 64, dtype, queries, keys, prefix=prefix, seed=11).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d", [(2, 2, 76), (3, 3, 41), (8, 1, 128), (2, 1, 256)])
def test_shared_prefix_head_widths(H, Hk, d, dtype):
    Packed(H, Hk, d, dtype, [1, 1, 1], [5, 0, 70], prefix=130, seed=12, gap=3).check()
    Packed(H, Hk, d, dtype, [17, 1, 140], [17, 40, 140], prefix=130, seed=13).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d", [(4, 2, 64), (2, 2, 128), (2, 2, 76), (1, 1, 41), (2, 1, 256)])
def test_shared_prefix_in_common_tiles(H, Hk, d, dtype):
    """A prefix much longer than the rows: rows of several sequences share tiles over it, and the own keys are parts of their own."""
    Packed(H, Hk, d, dtype, [20, 1, 7, 30], [20, 1, 9, 300], prefix=2000, seed=24).check()
    Packed(H, Hk, d, dtype, [20, 0, 33, 2], [5, 4, 0, 2], prefix=2000, seed=25, gap=2).check()


def test_prefix_equals_one_sequence_that_holds_it():
    """A shared prefix in front of one sequence is that sequence with a longer cache."""
    p = Packed(4, 2, 64, "f32", [30], [40], prefix=100, seed=14)
    a = p.run()
    b = Packed(4, 2, 64, "f32", [30], [140], seed=14)
    b.q, b.k, b.v = p.q, torch.cat((p.kp, p.k)), torch.cat((p.vp, p.v))
    c = b.run()
    close("O", a["O"], c["O"].double().cpu(), "f32")
    close("lse", a["lse"], c["lse"].double().cpu(), "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_sequences(dtype):
    """More sequences than one probe of the slot search tells apart (64 and 64 x 64)."""
    lens = [(i * 7) % 5 for i in range(4500)]
    p = Packed(2, 1, 8, dtype, lens, seed=15)
    p.check(backward=True)
    Packed(2, 1, 8, dtype, [1] * 300, [(i * 11) % 40 for i in range(300)], seed=16).check()


def test_infinite_and_large_logits():
    """Scores near the type's end, and a key whose score is -inf everywhere."""
    p = Packed(2, 2, 64, "bf16", [70, 1], [70, 200], seed=17, spread=30.0)
    got, ref = p.run(), p.reference()
    assert torch.isfinite(got["O"].float()).all()
    close("lse", got["lse"], ref["lse"], "f32")
    p = Packed(1, 1, 64, "f32", [3], [70], seed=18)
    p.q[:, :, 0], p.k[:, :, 0] = 1.0, 0.0
    p.k[5, 0, 0] = NEG
    got = p.run()
    p.k[5, 0, 0] = -1e30
    close("O", got["O"], p.reference()["O"], "f32")


@pytest.mark.parametrize("case", ["chunks", "tiles", "prefix", "prefix tiles"])
def test_nan_in_a_query_stays(case):
    """A query of NaN gives NaN, however its keys are split, and touches no other row."""
    p = {"chunks": lambda: Packed(4, 2, 64, "bf16", [1, 1, 1], [3000, 2, 500], seed=26), "tiles": lambda: Packed(2, 2, 64, "bf16", [40], [3001], seed=27),
         "prefix": lambda: Packed(4, 2, 64, "bf16", [1, 1, 1], [30, 2, 50], prefix=900, seed=28),
         "prefix tiles": lambda: Packed(4, 2, 64, "bf16", [20, 10], prefix=3000, seed=29)}[case]()
    a = p.run()
    row = p.q.shape[0] - 1
    p.q[row, 1, 3] = float("nan")
    b = p.run()
    assert torch.isnan(b["O"][row, 1]).all() and torch.isnan(b["lse"][1, row])
    for t in (a, b):
        t["O"][row, 1], t["lse"][1, row] = 0, 0
    assert torch.equal(a["O"], b["O"]) and torch.equal(a["lse"], b["lse"])


@pytest.mark.parametrize("H,Hk,d,queries,keys,prefix,causal,fused", [
    (48, 12, 128, [4096, 1, 300], None, 0, 1, False), (64, 64, 128, [4100, 77], [4100, 4500], 0, 1, False), (48, 48, 100, [4097], None, 0, 1, True),
    (33, 33, 101, [6000, 500], [6100, 100], 0, 1, False), (64, 16, 128, [5000], [3900], 300, 1, False), (16, 16, 128, [12300], [4200], 0, 0, False)])
def test_long_rows_in_tall_tiles(H, Hk, d, queries, keys, prefix, causal, fused):
    """Enough long rows for tiles of 256: every head of some, against float64 (one head at a time on the GPU)."""
    keys = queries if keys is None else keys
    p = Packed(H, Hk, d, "bf16", queries, keys, causal, prefix, seed=30, fused=fused)
    got = p.run()
    w = lambda t: t.cuda().double()
    for i, (n, m) in enumerate(zip(queries, keys)):
        qs, ks = slice(p.qoff[i], p.qoff[i] + n), slice(p.koff[i], p.koff[i] + m)
        hidden = torch.arange(m, device="cuda")[None] > (m - n) + torch.arange(n, device="cuda")[:, None] if causal else torch.zeros(n, m, dtype=torch.bool, device="cuda")
        if prefix:
            hidden = torch.cat((torch.zeros(n, prefix, dtype=torch.bool, device="cuda"), hidden), 1)
        for h in sorted({0, H // 2, H - 1}):
            hk = h // (H // Hk)
            k, v = w(p.k[ks, hk]), w(p.v[ks, hk])
            if prefix:
                k, v = torch.cat((w(p.kp[:, hk]), k)), torch.cat((w(p.vp[:, hk]), v))
            s = (w(p.q[qs, h]) @ k.t().contiguous() * p.scale).masked_fill_(hidden, NEG)
            close("lse", got["lse"][h, qs], torch.logsumexp(s, 1).cpu(), "f32")
            close("O", got["O"][qs, h], (torch.nan_to_num(torch.softmax(s, 1)) @ v).cpu(), "bf16")


@pytest.mark.parametrize("H,Hk,d", [(2, 2, 64), (4, 1, 128), (1, 1, 256)])
def test_more_parts_than_lanes(H, Hk, d):
    """A token over so many chunks of keys that the joining wave takes their sums in several rounds."""
    Packed(H, Hk, d, "bf16", [1], [20000], seed=33).check()
    Packed(H, Hk, d, "f32", [1, 2], [17001, 300], seed=34).check()


def test_backward_in_ranges_of_rows():
    """Few key tiles and many rows: dK and dV from several ranges of rows."""
    Packed(8, 2, 128, "bf16", [700, 5], seed=35).check(backward=True)
    Packed(6, 1, 76, "bf16", [500], [300], seed=36, causal=0).check(backward=True)


def test_backward_that_keeps_no_score_gradients():
    """More keys and rows than score gradients are kept for: dQ computes them again."""
    p = Packed(4, 1, 32, "bf16", [300, 1], seed=37)
    p.k, p.v = (torch.cat((t, torch.full((1 << 20, 1, 32), 3.0, dtype=t.dtype))) for t in (p.k, p.v))   # rows of no sequence
    plan = binding.make_attention(p.q, p.k, p.v, p.q, 2, 300, 300)
    assert binding.switchhead_attention_workspace_bytes(plan, True) < p.k.shape[0] * 1200 * 2
    p.check(backward=True)


def test_calls_on_two_streams():
    """Two calls at once, each with its stream and workspace."""
    ps = [Packed(8, 2, 128, "bf16", [130, 257, 1, 64], seed=31), Packed(4, 4, 64, "bf16", [1] * 5, [3000, 5, 70, 900, 1], seed=32)]
    alone = [p.run() for p in ps]
    streams, runs = [torch.cuda.Stream() for _ in ps], []
    for p, s in zip(ps, streams):
        q, k, v = p.device()
        O, off = torch.zeros_like(q), [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (p.qoff, p.koff)]
        plan = binding.make_attention(q, k, v, O, len(p.nq), max(p.nq), max(p.nk))
        runs.append((s, plan, q, k, v, *off, O, torch.empty(binding.switchhead_attention_workspace_bytes(plan), dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(3):
        for s, plan, q, k, v, qo, ko, O, ws in runs:
            with torch.cuda.stream(s):
                binding.switchhead_attention_forward(plan, q, k, v, qo, ko, O, None, ws)
    torch.cuda.synchronize()
    for a, r in zip(alone, runs):
        assert torch.equal(a["O"], r[7])


def test_bounds_on_the_lengths():
    """Larger bounds than the lengths only split the work otherwise; smaller ones cut the sequences."""
    p = Packed(4, 2, 64, "f32", [1, 1, 1], [700, 3, 2500], seed=19)
    ref = p.reference()
    for mk in (2500, 3203, 100000):
        got = p.run(max_k=mk)
        close("O", got["O"], ref["O"], "f32")
        close("lse", got["lse"], ref["lse"], "f32")
    p = Packed(4, 2, 64, "f32", [40, 2, 60], [700, 3, 2500], seed=20)
    for mq, mk in ((5, 2500), (60, 200), (5, 90)):
        got = p.run(backward=True, max_q=mq, max_k=mk)
        cut = Packed(4, 2, 64, "f32", [min(n, mq) for n in p.nq], [min(n, mk) for n in p.nk], seed=20)
        cut.q, cut.k, cut.v, cut.dO, cut.qoff, cut.koff = p.q, p.k, p.v, p.dO, p.qoff, p.koff
        ref = cut.reference(backward=True)
        for n in ("O", "lse", "dQ", "dK", "dV"):   # 777: rows that were cut off are left
            close(n, got[n], ref[n], "f32")


def test_offsets_out_of_range_stay_inside():
    """Offsets and lengths that lie are cut to the tensors' rows: nothing outside is touched (rows in front of and behind the views)."""
    guard = torch.full((64, 4, 64), 5.0, device="cuda", dtype=torch.bfloat16)
    O = guard[16:48]
    q, k = torch.randn(32, 4, 64, device="cuda").bfloat16(), torch.randn(32, 4, 64, device="cuda").bfloat16()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    plan = binding.make_attention(q, k, k, O, 3, 32, 32)
    ws = torch.empty(binding.switchhead_attention_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    for off, lens in (([-5, 10, 20, 400], None), ([0, 8, 16, 24], [100, -3, 1000]), ([2000000000, 2000000000, -2000000000, 7], None)):
        binding.switchhead_attention_forward(plan, q, k, k, i32(off), i32(off), O, None, ws, None if lens is None else i32(lens), None if lens is None else i32(lens))
        torch.cuda.synchronize()
        assert torch.all(guard[:16] == 5.0) and torch.all(guard[48:] == 5.0)


def test_results_repeat():
    p = Packed(8, 2, 128, "bf16", [130, 257, 1, 64], seed=21)
    a, b = p.run(backward=True), p.run(backward=True, ws_fill=3)
    assert all(torch.equal(a[n], b[n]) for n in a)
    p = Packed(8, 2, 128, "bf16", [1, 1], [3000, 2], prefix=500, seed=22)
    a, b = p.run(), p.run(ws_fill=3)
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_gradient_against_differences():
    """dQ, dK, dV against central differences of <O, dO> computed by the operator itself."""
    p = Packed(2, 1, 32, "f32", [5, 9], seed=23)
    got = p.run(backward=True)
    g = torch.Generator().manual_seed(1)
    for name in ("q", "k", "v"):
        t = getattr(p, name)
        kept, step = t.clone(), torch.randn(t.shape, generator=g)
        vals = []
        for e in (0.02, -0.02):   # fp32 outputs: error e^2 of the third derivative against 2^-24 / e of the values
            setattr(p, name, kept + e * step)
            vals.append(float((p.run()["O"].double().cpu() * p.dO.double()).sum()))
        setattr(p, name, kept)
        ref = (vals[0] - vals[1]) / 0.04
        mine = float((got["d" + name.upper()].double().cpu() * step.double()).sum())
        assert abs(mine - ref) <= 5e-3 * max(abs(ref), 1.0), (name, mine, ref)


def test_captured_and_replayed_with_other_lengths():
    """A captured call reads the lengths from the device: replays follow them."""
    torch.manual_seed(0)
    q, k, v = (torch.randn(40, 4, 64, device="cuda").bfloat16() for _ in range(3))
    dO = torch.randn_like(q)
    O, dq, dk, dv = (torch.zeros_like(q) for _ in range(4))
    lse = torch.zeros(4, 40, device="cuda")
    off = torch.tensor([0, 10, 25, 40], dtype=torch.int32, device="cuda")
    plan = binding.make_attention(q, k, v, O, 3, 40, 40)
    ws = torch.empty(max(binding.switchhead_attention_workspace_bytes(plan, b) for b in (False, True)), dtype=torch.uint8, device="cuda")

    def step():
        binding.switchhead_attention_forward(plan, q, k, v, off, off, O, lse, ws)
        binding.switchhead_attention_backward(plan, q, k, v, O, dO, lse, off, off, dq, dk, dv, ws)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for lens in ([0, 10, 25, 40], [0, 40, 40, 40], [0, 1, 2, 40]):
        off.copy_(torch.tensor(lens, dtype=torch.int32))
        for t in (O, dq, dk, dv):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        again = [t.clone() for t in (O, lse, dq, dk, dv)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, (O, lse, dq, dk, dv)))


def test_long_rows_past_32_bits():
    """Key rows whose byte offsets pass 2^32: a cache of 2.2 million rows of 8 heads of 128."""
    rows, d = 2_200_000, 128
    k = torch.empty(rows, 8, d, device="cuda", dtype=torch.bfloat16)
    v = torch.empty(rows, 8, d, device="cuda", dtype=torch.bfloat16)
    n = 200
    torch.manual_seed(3)
    kk, vv = torch.randn(n, 8, d).bfloat16(), torch.randn(n, 8, d).bfloat16()
    k[rows - n:], v[rows - n:] = kk.cuda(), vv.cuda()
    for queries in (1, 60):
        q = torch.randn(queries, 8, d).bfloat16()
        O = torch.empty(queries, 8, d, device="cuda", dtype=torch.bfloat16)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        plan = binding.make_attention(q.cuda(), k, v, O, 1, queries, n)
        ws = torch.empty(binding.switchhead_attention_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
        qd = q.cuda()
        binding.switchhead_attention_forward(plan, qd, k, v, i32([0, queries]), i32([rows - n, rows]), O, None, ws)
        torch.cuda.synchronize()
        ref = oracle(q.double(), kk.double(), vv.double(), queries, n, 1, 1, 1 / math.sqrt(d))[0]
        close("O", O, ref, "bf16")


# ---- norms and rotation ----------------------------------------------------------------------------------------------------
def norm_oracle(x, w, pos, rope_dim, eps, theta, dY=None):
    x = x.double()
    d = x.shape[-1]
    w = torch.ones(d, dtype=torch.float64) if w is None else w.double()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    ang = pos.double()[:, None] * torch.tensor([theta ** (-2.0 * i / rope_dim) for i in range(rope_dim // 2)], dtype=torch.float64)
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]

    def turn(t, sign):
        t = t.clone()
        a, b = t[..., 0:rope_dim:2].clone(), t[..., 1:rope_dim:2].clone()
        t[..., 0:rope_dim:2], t[..., 1:rope_dim:2] = a * c - sign * b * s, sign * a * s + b * c
        return t

    y = turn(x * r * w, 1)
    if dY is None:
        return y, None, None
    dn = turn(dY.double(), -1)
    g = dn * w
    return y, r * (g - x * r * r * (g * x).mean(-1, keepdim=True)), (dn * x * r).sum((0, 1))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,H,Hk,d,rope_dim", [(1, 1, 1, 2, 2), (5, 4, 4, 128, 128), (130, 8, 2, 64, 32), (33, 2, 2, 76, 76), (17, 3, 3, 41, 40),
                                                    (9, 5, 1, 80, 0), (70, 2, 1, 256, 256), (3, 2, 0, 100, 50), (2100, 1, 1, 8, 8)])
def test_norms_and_rotation(tokens, H, Hk, d, rope_dim, dtype):
    """Forward and gradients over head widths, partly turned heads, positions far out and negative, fused views."""
    g = torch.Generator().manual_seed(tokens)
    t = (torch.randn(tokens, H + Hk + 1, d, generator=g) * torch.exp(torch.randn(tokens, H + Hk + 1, 1, generator=g))).to(DT[dtype])
    dt = torch.randn(tokens, H + Hk, d, generator=g).to(DT[dtype])
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(DT[dtype]) for _ in range(2)]
    pos = torch.randint(-1000, 2_000_000, (tokens,), generator=g, dtype=torch.int32)
    dev = t.cuda()
    Q, K = dev[:, :H], dev[:, H:H + Hk] if Hk else None
    Y = torch.full((tokens, H + Hk, d), 7.0, dtype=t.dtype, device="cuda")
    YQ, YK = Y[:, :H], Y[:, H:] if Hk else None
    plan = binding.make_qk_norm(Q, K, YQ, YK, rope_dim, eps=1e-5, theta=500.0)
    wq, wk, p = w[0].cuda(), w[1].cuda(), pos.cuda()
    binding.switchhead_qk_norm_rope_forward(plan, Q, K, wq, wk, p, YQ, YK)
    grad = torch.full(dev.shape, 7.0, dtype=t.dtype, device="cuda")
    dw = [torch.empty(d, device="cuda") for _ in range(2)]
    ws = torch.full((binding.switchhead_qk_norm_workspace_bytes(plan),), 255, dtype=torch.uint8, device="cuda")
    dY = dt.cuda()
    binding.switchhead_qk_norm_rope_backward(plan, Q, K, wq, wk, p, dY[:, :H], dY[:, H:] if Hk else None, grad[:, :H], grad[:, H:H + Hk] if Hk else None,
                                             dw[0], dw[1], ws)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(((0, H), (H, H + Hk))):
        if a == b:
            continue
        y, dx, dwr = norm_oracle(t[:, a:b], w[i], pos, rope_dim, 1e-5, 500.0, dt[:, a:b])
        close("y", Y[:, a:b], y, dtype)
        close("dx", grad[:, a:b], dx, dtype, scale=max(float(dx.norm()), 1e-2 * math.sqrt(dx.numel())))
        close("dw", dw[i], dwr, "f32", scale=max(float(dwr.norm()), math.sqrt(tokens * (b - a) * d)))
    assert torch.all(grad[:, H + Hk:] == 7.0)


def test_norm_in_place_ones_and_default_positions():
    x = torch.randn(40, 4, 64, device="cuda")
    host = x.cpu()
    plan = binding.make_qk_norm(x, None, x, None, 64)
    binding.switchhead_qk_norm_rope_forward(plan, x, None, None, None, None, x, None)
    torch.cuda.synchronize()
    y, _, _ = norm_oracle(host, None, torch.arange(40), 64, 1e-6, 10000.0)
    close("y", x, y, "f32")


def test_zero_rows_of_x():
    """A row of zeros has norm sqrt(eps): zeros out, finite gradient; eps 0 with nonzero rows."""
    x = torch.zeros(3, 2, 32, device="cuda")
    x[1] = torch.randn(2, 32, device="cuda")
    y = torch.empty_like(x)
    plan = binding.make_qk_norm(x, None, y, None, 32, eps=1e-6)
    binding.switchhead_qk_norm_rope_forward(plan, x, None, None, None, None, y, None)
    dx, dw = torch.empty_like(x), torch.empty(32, device="cuda")
    ws = torch.empty(binding.switchhead_qk_norm_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    dy = torch.randn_like(x)
    binding.switchhead_qk_norm_rope_backward(plan, x, None, None, None, None, dy, None, dx, None, dw, None, ws)
    torch.cuda.synchronize()
    ry, rdx, rdw = norm_oracle(x.cpu(), None, torch.arange(3), 32, 1e-6, 10000.0, dy.cpu())
    close("y", y, ry, "f32")
    close("dx", dx, rdx, "f32")
    close("dw", dw, rdw, "f32")


def test_norm_then_attention_then_back():
    """The operators in a row, as a training step and as decoding over what it left: norms and rotation, attention, both gradients;
    then single tokens over the turned keys give the packed call's last rows."""
    torch.manual_seed(1)
    lens, H, Hk, d = [70, 1, 129], 4, 2, 64
    N = sum(lens)
    qkv = torch.randn(N, H + 2 * Hk, d).bfloat16()
    w = [(1 + 0.1 * torch.randn(d)).bfloat16() for _ in range(2)]
    pos = torch.cat([torch.arange(n) for n in lens]).int()
    off = torch.tensor([0, 70, 71, 200], dtype=torch.int32, device="cuda")
    dO = torch.randn(N, H, d).bfloat16()
    t = qkv.cuda()
    Q, K, V = t[:, :H], t[:, H:H + Hk], t[:, H + Hk:]
    YQ, YK = torch.empty(N, H, d, dtype=t.dtype, device="cuda"), torch.empty(N, Hk, d, dtype=t.dtype, device="cuda")
    nplan = binding.make_qk_norm(Q, K, YQ, YK, d)
    wq, wk, p = w[0].cuda(), w[1].cuda(), pos.cuda()
    binding.switchhead_qk_norm_rope_forward(nplan, Q, K, wq, wk, p, YQ, YK)
    O, lse = torch.empty_like(YQ), torch.empty(H, N, device="cuda")
    aplan = binding.make_attention(YQ, YK, V, O, 3, 129, 129)
    ws = torch.empty(max(binding.switchhead_attention_workspace_bytes(aplan, b) for b in (False, True)), dtype=torch.uint8, device="cuda")
    binding.switchhead_attention_forward(aplan, YQ, YK, V, off, off, O, lse, ws)
    grad = torch.empty_like(t)
    dYQ, dYK = torch.empty_like(YQ), torch.empty_like(YK)
    binding.switchhead_attention_backward(aplan, YQ, YK, V, O, dO.cuda(), lse, off, off, dYQ, dYK, grad[:, H + Hk:], ws)
    nws = torch.empty(binding.switchhead_qk_norm_workspace_bytes(nplan), dtype=torch.uint8, device="cuda")
    dw = [torch.empty(d, device="cuda") for _ in range(2)]
    binding.switchhead_qk_norm_rope_backward(nplan, Q, K, wq, wk, p, dYQ, dYK, grad[:, :H], grad[:, H:H + Hk], dw[0], dw[1], nws)
    torch.cuda.synchronize()
    # autograd over an independent float64 form
    x = qkv.double().requires_grad_(True)
    ww = [v.double().requires_grad_(True) for v in w]
    ang = pos.double()[:, None] * torch.tensor([10000.0 ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64)

    def turned(a):
        z = torch.view_as_complex(a.reshape(N, -1, d // 2, 2)) * torch.polar(torch.ones_like(ang), ang)[:, None]
        return torch.view_as_real(z).reshape(N, -1, d)

    yq = turned(x[:, :H] / torch.sqrt((x[:, :H] ** 2).mean(-1, keepdim=True) + 1e-6) * ww[0])
    yk = turned(x[:, H:H + Hk] / torch.sqrt((x[:, H:H + Hk] ** 2).mean(-1, keepdim=True) + 1e-6) * ww[1])
    outs, a = [], 0
    for n in lens:
        q, k, v = yq[a:a + n].transpose(0, 1), yk[a:a + n].repeat_interleave(H // Hk, 1).transpose(0, 1), x[a:a + n, H + Hk:].repeat_interleave(H // Hk, 1).transpose(0, 1)
        s = q @ k.transpose(1, 2) / math.sqrt(d) + torch.full((n, n), NEG, dtype=torch.float64).triu(1)
        outs.append((torch.softmax(s, -1) @ v).transpose(0, 1))
        a += n
    ref = torch.cat(outs)
    ref.backward(dO.double())
    # turned queries, keys and their gradients are rounded to bf16 on the way: two more roundings than an operator by itself
    for name, got, want in (("O", O, ref.detach()), ("dqkv", grad, x.grad), ("dw_Q", dw[0], ww[0].grad), ("dw_K", dw[1], ww[1].grad)):
        err = float((got.double().cpu() - want).norm() / want.norm())
        print(name, "%.2e" % err)
        assert err < 2 * REL["bf16"], name
    last = torch.tensor([69, 70, 199], device="cuda")
    q1 = YQ[last].contiguous()
    o1 = torch.empty_like(q1)
    dplan = binding.make_attention(q1, YK, V, o1, 3, 1, 129)
    ws = torch.empty(binding.switchhead_attention_workspace_bytes(dplan), dtype=torch.uint8, device="cuda")
    binding.switchhead_attention_forward(dplan, q1, YK, V, torch.arange(4, dtype=torch.int32, device="cuda"), off, o1, None, ws)
    torch.cuda.synchronize()
    close("decoded", o1, O[last].double().cpu(), "bf16")
