"""Calls of the attention and norm operators at the edges of what their description allows, on the GPU: offsets that lie, unusual numbering of the
work, scales, padding."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2312_07987_amd import binding
from test_gpu_attention_ops import Packed, close, norm_oracle

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Guarded:
    """A tensor in the middle of a larger one that holds 5."""

    def __init__(self, shape, dtype, pad=40):
        self.all = torch.full((shape[0] + 2 * pad,) + tuple(shape[1:]), 5.0, dtype=dtype, device="cuda")
        self.pad, self.t = pad, self.all[pad:pad + shape[0]]

    def check(self):
        assert torch.all(self.all[:self.pad] == 5.0) and torch.all(self.all[self.pad + self.t.shape[0]:] == 5.0)


LYING = [
    [0, 1152, 0, 1152],                                   # the second sequence's slots lie behind the third's
    [1152, 700, 300, 0], [0, 0, 0, 1152], [500, 2000000000, -2000000000, 600], [1152, 0, 1152, 0], [-5, 10, 2000, 3],
    [(i * 397) % 1153 for i in range(140)],               # more sequences than one probe tells apart
]


@pytest.mark.parametrize("dtype,H,Hk,d", [("bf16", 4, 2, 64), ("f32", 4, 2, 32), ("bf16", 2, 1, 128), ("bf16", 2, 2, 256)])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("most", [1152, 1])
def test_falling_offsets_stay_inside(dtype, H, Hk, d, causal, most):
    """Whatever the offsets hold, forward and backward end, and touch nothing outside the tensors.  most 1: single tokens, keys in chunks."""
    n = 1152
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda h: torch.randn(n, h, d, generator=g, device="cuda").to(DT[dtype])
    q, k, v, dO = rnd(H), rnd(Hk), rnd(Hk), rnd(H)
    for off in LYING:
        print(off[:4], flush=True)
        O, dQ, dK, dV = (Guarded((n, h, d), DT[dtype]) for h in (H, H, Hk, Hk))
        lse = torch.full((H + 2, n), 5.0, device="cuda")
        plan = binding.make_attention(q, k, v, O.t, len(off) - 1, most, n, causal)
        ws = torch.zeros(max(binding.switchhead_attention_workspace_bytes(plan, b) for b in (False, True)), dtype=torch.uint8, device="cuda")
        binding.switchhead_attention_forward(plan, q, k, v, i32(off), i32(off), O.t, lse[1:-1], ws)
        torch.cuda.synchronize()
        binding.switchhead_attention_backward(plan, q, k, v, O.t, dO, lse[1:-1], i32(off), i32(off), dQ.t, dK.t, dV.t, ws)
        torch.cuda.synchronize()
        for t in (O, dQ, dK, dV):
            t.check()
        assert torch.all(lse[0] == 5.0) and torch.all(lse[-1] == 5.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_falling_offsets_behind_a_prefix(dtype):
    n, H, Hk, d = 1152, 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda rows, h: torch.randn(rows, h, d, generator=g, device="cuda").to(DT[dtype])
    q, k, kp = rnd(n, H), rnd(n, Hk), rnd(700, Hk)
    for most in (1, 200, n):
        for off in LYING:
            print(most, off[:4], flush=True)
            O = Guarded((n, H, d), DT[dtype])
            plan = binding.make_attention(q, k, k, O.t, len(off) - 1, most, n, 1, kp, kp)
            ws = torch.zeros(binding.switchhead_attention_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
            binding.switchhead_attention_forward(plan, q, k, k, i32(off), i32(off), O.t, None, ws, K_prefix=kp, V_prefix=kp)
            torch.cuda.synchronize()
            O.check()


def by_slot(lengths, group, kv_heads, tile=128):
    """The sequences are so many and the longest so long that a launch under a causal mask numbers its tiles one sequence after the other, not by level."""
    tiles = -(-max(lengths) * group // tile)
    return tiles * len(lengths) > 2 * (sum(lengths) * group // tile + len(lengths)) + 1024 // kv_heads


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 8, 76), (4, 4, 128), (4, 2, 32)])
@pytest.mark.parametrize("place", ["front", "middle", "end"])
def test_a_long_document_among_many_short_ones(H, Hk, d, dtype, place):
    """Causal training batches whose tiles, of rows and of keys, are numbered by slot."""
    lens = [(i * 5) % 4 for i in range(300)]
    lens.insert(dict(front=0, middle=150, end=300)[place], 700)
    assert by_slot(lens, H // Hk, Hk) and by_slot(lens, 1, Hk)
    Packed(H, Hk, d, dtype, lens, seed=40).check(backward=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.02, 0.7])
def test_a_scale_of_its_own(dtype, scale):
    for p in (Packed(4, 2, 64, dtype, [40, 1, 130], seed=41), Packed(2, 1, 76, dtype, [60, 5], [90, 300], seed=42, causal=0)):
        p.scale = scale
        p.check(backward=True, scale=scale)
    for p in (Packed(4, 2, 64, dtype, [1, 1], [700, 30], seed=43), Packed(4, 2, 64, dtype, [1, 5], [70, 30], prefix=900, seed=44)):
        p.scale = scale
        p.check(scale=scale)


def test_gradients_when_every_key_is_visible_and_none_is_queried():
    """Keys without queries get gradients of zero, queries without keys too; whole launches without rows on one side."""
    for nq, nk in (([0, 0], [70, 5]), ([70, 5], [0, 0]), ([0, 3], [9, 0])):
        for causal in (0, 1):
            for dtype in ("f32", "bf16"):
                Packed(4, 2, 64, dtype, nq, nk, causal=causal, seed=45).check(backward=True, max_q=max(max(nq), 1), max_k=max(max(nk), 1))


@pytest.mark.parametrize("H,Hk,d", [(4, 1, 128), (4, 1, 76)])
def test_more_score_gradients_than_are_kept(H, Hk, d):
    """Wide heads whose score gradients would take more than 2 GiB: dQ works the scores out again.  Narrow heads keep none at any size."""
    p = Packed(H, Hk, d, "bf16", [300, 1, 33], seed=46)
    few = binding.make_attention(p.q, p.k, p.v, p.q, 3, 300, 300)
    assert binding.switchhead_attention_workspace_bytes(few, True) >= p.k.shape[0] * 1200 * 2
    p.check(backward=True)
    p.k, p.v = (torch.cat((t, torch.full((1 << 20, Hk, d), 3.0, dtype=t.dtype))) for t in (p.k, p.v))   # rows of no sequence
    many = binding.make_attention(p.q, p.k, p.v, p.q, 3, 300, 300)
    assert binding.switchhead_attention_workspace_bytes(many, True) < p.k.shape[0] * 1200 * 2
    p.check(backward=True)
    n = Packed(4, 1, 64, "bf16", [1200], seed=47)
    plan = binding.make_attention(n.q, n.k, n.v, n.q, 1, 1200, 1200)
    assert binding.switchhead_attention_workspace_bytes(plan, True) < 1200 * 4800 * 2


def laid(t, layout):
    """t's values on the GPU, head by head (rows of all tokens of a head behind each other), or beginning one element behind an aligned address."""
    if layout == "by head":
        return t.transpose(0, 1).contiguous().cuda().transpose(0, 1)
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    out = flat[1:].view(t.shape)
    out.copy_(t)
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["by head", "odd address"])
@pytest.mark.parametrize("H,Hk,d", [(4, 2, 64), (2, 2, 128), (2, 1, 76)])
def test_other_layouts(H, Hk, d, layout, dtype):
    p = Packed(H, Hk, d, dtype, [70, 1, 130], seed=48)
    ref = p.reference(backward=True)
    bounds = ref.pop("bounds")
    q, k, v, dO = (laid(t, layout) for t in (p.q, p.k, p.v, p.dO))
    O, dq, dk, dv = (laid(torch.full(t.shape, 777.0, dtype=t.dtype), layout) for t in (p.q, p.q, p.k, p.v))
    lse, off = torch.empty(H, p.q.shape[0], device="cuda"), i32(p.qoff)
    plan = binding.make_attention(q, k, v, O, 3, 130, 130)
    ws = torch.full((max(binding.switchhead_attention_workspace_bytes(plan, b) for b in (False, True)),), 255, dtype=torch.uint8, device="cuda")
    binding.switchhead_attention_forward(plan, q, k, v, off, off, O, lse, ws)
    binding.switchhead_attention_backward(plan, q, k, v, O, dO, lse, off, off, dq, dk, dv, ws)
    torch.cuda.synchronize()
    close("O", O, ref["O"], dtype)
    close("dV", dv, ref["dV"], dtype)
    for n, t in (("dQ", dq), ("dK", dk)):
        assert float(((t.double().cpu() - ref[n]).abs() - bounds[n]).max()) <= 0, n
    one = Packed(H, Hk, d, dtype, [1, 1, 1], [70, 1, 300], seed=49)   # single tokens
    q, k, v = (laid(t, layout) for t in (one.q, one.k, one.v))
    O = laid(torch.zeros_like(one.q), layout)
    plan = binding.make_attention(q, k, v, O, 3, 1, 300)
    ws = torch.empty(binding.switchhead_attention_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    binding.switchhead_attention_forward(plan, q, k, v, i32(one.qoff), i32(one.koff), O, None, ws)
    torch.cuda.synchronize()
    close("token", O, one.reference()["O"], dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["by head", "odd address"])
@pytest.mark.parametrize("tokens", [1, 37])
def test_norms_of_other_layouts_in_place(tokens, layout, dtype):
    """Forward into the input and gradients into the upstream gradient, which lies as they do."""
    g = torch.Generator().manual_seed(50)
    x, dy = (torch.randn(tokens, 4, 64, generator=g).to(DT[dtype]) for _ in range(2))
    dx, dw = laid(dy, layout), torch.empty(64, device="cuda")
    kept, y = laid(x, layout), laid(x, layout)
    plan = binding.make_qk_norm(kept, None, y, None, 32)
    binding.switchhead_qk_norm_rope_forward(plan, y, None, None, None, None, y, None)
    ws = torch.empty(binding.switchhead_qk_norm_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    binding.switchhead_qk_norm_rope_backward(plan, kept, None, None, None, None, dx, None, dx, None, dw, None, ws)
    torch.cuda.synchronize()
    ry, rdx, rdw = norm_oracle(x, None, torch.arange(tokens), 32, 1e-6, 10000.0, dy)
    close("y", y, ry, dtype)
    close("dx", dx, rdx, dtype)
    close("dw", dw, rdw, "f32", scale=max(float(rdw.norm()), math.sqrt(tokens * 4 * 64)))


@pytest.mark.parametrize("H,Hk,d,queries,keys,causal", [(2, 2, 64, [20] * 10, None, 1), (2, 2, 76, [20, 256, 33, 1, 60, 110], None, 1), (8, 2, 128, [30, 7, 200], None, 1),
                                                       (2, 1, 256, [33, 40], None, 1), (4, 4, 41, [25, 3], None, 1), (4, 2, 64, [50, 9, 70], [20, 32, 31], 0),
                                                       (4, 2, 32, [40, 20, 3, 50], [60, 12, 30, 50], 1)])
def test_gradients_are_off_by_two_roundings_alone(H, Hk, d, queries, keys, causal):
    """bf16: dQ and dK carry the roundings of dS, once before its products, and of the result, and nothing else that counts.  How large these two are is worked out in
    float64 for the same tensors; the rest (dS from other sums in fp32, rows of more than 32 keys whose <dO, O> is of rounded rows) adds less than a tenth
    of that where most rows see few keys: two independent errors of 1 and 0.4 make 1.08."""
    keys = queries if keys is None else keys
    p = Packed(H, Hk, d, "bf16", queries, keys, causal, seed=60)
    got, ref, bf = p.run(backward=True), p.reference(backward=True), lambda t: t.bfloat16().double()
    alone = {n: torch.zeros_like(ref[n]) for n in ("dQ", "dK")}
    for i, (n, m) in enumerate(zip(queries, keys)):
        qs, ks = slice(p.qoff[i], p.qoff[i] + n), slice(p.koff[i], p.koff[i] + m)
        hidden = torch.arange(m)[None] > (m - n) + torch.arange(n)[:, None] if causal else torch.zeros(n, m, dtype=torch.bool)
        for h in range(H):
            q, k, v, dO = (t.double() for t in (p.q[qs, h], p.k[ks, h // (H // Hk)], p.v[ks, h // (H // Hk)], p.dO[qs, h]))
            P = torch.nan_to_num(torch.softmax((q @ k.t() * p.scale).masked_fill(hidden, -math.inf), 1))
            dP = dO @ v.t()
            dS = bf(P * (dP - (P * dP).sum(1, keepdim=True)))
            alone["dQ"][qs, h] = dS @ k * p.scale
            alone["dK"][ks, h // (H // Hk)] += dS.t() @ q * p.scale
    for n, t in alone.items():
        two = float((bf(t) - ref[n]).norm())
        err = float((got[n].double().cpu() - ref[n]).norm())
        print(n, "%.3e of %.3e: %.3f" % (err, two, err / two), flush=True)
        assert err <= 1.08 * two, n
