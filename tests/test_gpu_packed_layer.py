"""The layer over packed sequences (norms of queries and keys, rotary positions, a shared prefix) on the GPU: against an independent float64
form by torch.autograd, one sequence at a time, and against the plain layer's own calls for the same sequences.

The bars are the layer's: the largest error of a tensor over its largest element at most 2e-2 (bf16 storage) and 1e-4 (fp32)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2312_07987_amd import binding
from paper_2312_07987_amd.inputs import make_inputs
from paper_2312_07987_amd.runner import DeviceLayer

pytestmark = pytest.mark.gpu
BAR = {"f32": 1e-4, "bf16": 2e-2}
NAMES = ("W_Q", "W_K", "W_V", "W_O", "W_S", "W_D")


def turned(a, pos, d):
    half = d // 2
    ang = pos.double()[:, None] * torch.tensor([10000.0 ** (-2.0 * i / (2 * half)) for i in range(half)], dtype=torch.float64)
    z = torch.view_as_complex(a[..., :2 * half].reshape(a.shape[0], a.shape[1], half, 2).contiguous()) * torch.polar(torch.ones_like(ang), ang)[:, None]
    return torch.cat((torch.view_as_real(z).reshape(a.shape[0], a.shape[1], 2 * half), a[..., 2 * half:]), -1)


def reference(cfg, t, offsets, prefix, w_norm, eps):
    """y of the T - prefix rows, differentiable in the tensors of t (all float64)."""
    H, E, k, d = cfg["nheads"], cfg["E"], cfg["k"], cfg["d_head"]
    x = t["x"][0]
    N = x.shape[0]

    def gates(W, rows):
        z = (rows @ W).reshape(-1, H, E)
        top = torch.topk(z.detach(), k, -1).indices
        return torch.sigmoid(z) * torch.zeros_like(z).scatter(-1, top, 1.0)

    xq = x[prefix:]
    gS, gD = gates(t["W_S"], x), gates(t["W_D"] if t["W_D"] is not None else t["W_S"], xq)
    Q, K = torch.einsum("nd,hde->nhe", xq, t["W_Q"]), torch.einsum("nd,hde->nhe", x, t["W_K"])
    V = torch.einsum("nhe,nd,hedf->nhf", gS, x, t["W_V"])
    if w_norm:
        Q = Q / torch.sqrt((Q * Q).mean(-1, keepdim=True) + eps) * w_norm[0]
        K = K / torch.sqrt((K * K).mean(-1, keepdim=True) + eps) * w_norm[1]
    ctx = [torch.zeros(0, H, d, dtype=torch.float64)]
    at = 0
    for a, b in zip(offsets[:-1], offsets[1:]):
        ctx.append(torch.zeros(a - at, H, d, dtype=torch.float64))
        at = b
        n = b - a
        q, kk, v = Q[a:b], K[prefix + a:prefix + b], V[prefix + a:prefix + b]
        kp, vp = K[:prefix], V[:prefix]
        if cfg.get("rope"):
            own = prefix + torch.arange(n)
            q, kk, kp = turned(q, own, d), turned(kk, own, d), turned(kp, torch.arange(prefix), d)
        kk, v = torch.cat((kp, kk)), torch.cat((vp, v))
        s = torch.einsum("nhe,mhe->hnm", q, kk) / math.sqrt(d)
        if cfg["causal"]:
            hidden = torch.cat((torch.zeros(n, prefix, dtype=torch.bool), torch.ones(n, n, dtype=torch.bool).triu(1)), 1)
            s = s.masked_fill(hidden, -math.inf)
        ctx.append(torch.einsum("hnm,mhe->nhe", torch.softmax(s, -1), v))
    ctx.append(torch.zeros(N - prefix - at, H, d, dtype=torch.float64))
    return torch.einsum("nhe,nhf,hefd->nd", gD, torch.cat(ctx), t["W_O"])


def close(name, got, ref, dtype):
    got, ref = got.double().cpu(), ref.detach()
    err = float((got - ref).abs().max() / max(float(ref.abs().max()), 1e-30))
    print(name, "%.2e" % err, flush=True)
    assert err <= BAR[dtype], (name, err)


def run(cfg, lens, prefix=0, norm=False, lead=0, tail=0, backward=True, shared=False):
    """lead, tail: rows in front of the first and behind the last sequence that belong to none."""
    offsets = np.concatenate(([0], np.cumsum(lens))) + lead
    T = int(prefix + offsets[-1] + tail)
    cfg = dict(cfg, B=1, T=T, T_q=T - prefix if prefix else 0)
    host = make_inputs(cfg, seed=sum(lens) + prefix, shared_router=shared)
    layer = DeviceLayer(cfg, host)
    d = cfg["d_head"]
    g = torch.Generator().manual_seed(5)
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(layer.tdtype) for _ in range(2)] if norm else None
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    packing = binding.make_packing(off, max(max(lens), 1), *([v.cuda() for v in w] if norm else (None, None)), norm_eps=1e-5)
    ws = torch.empty(binding.switchhead_packed_workspace_bytes(layer.shape, packing), dtype=torch.uint8, device="cuda")
    ws.fill_(255)
    W = layer.W
    binding.switchhead_forward_packed(layer.shape, packing, layer.x, W["W_Q"], W["W_K"], W["W_V"], W["W_O"], W["W_S"], W["W_D"], None, None, layer.y, ws)
    dn = [torch.empty(d, device="cuda") for _ in range(2)]
    if backward:
        dW = layer.dW
        binding.switchhead_backward_packed(layer.shape, packing, layer.x, W["W_Q"], W["W_K"], W["W_V"], W["W_O"], W["W_S"], W["W_D"], layer.dy, ws, layer.dx,
                                           dW["W_Q"], dW["W_K"], dW["W_V"], dW["W_O"], dW["W_S"], dW["W_D"], layer.db_S, layer.db_D, *(dn if norm else (None, None)))
    torch.cuda.synchronize()
    t = {n: None if host.get(n) is None else torch.from_numpy(host[n]).double().requires_grad_(True) for n in ("x",) + NAMES}
    wn = [v.double().requires_grad_(True) for v in w] if norm else None
    y = reference(cfg, t, offsets.tolist(), prefix, wn, 1e-5)
    close("y", layer.y[0], y, cfg["dtype"])
    if backward:
        y.backward(torch.from_numpy(host["dy"][0]).double())
        close("dx", layer.dx, t["x"].grad, cfg["dtype"])
        for n in NAMES:
            if t[n] is not None:
                close("d" + n, layer.dW[n], t[n].grad, cfg["dtype"])
        if norm:
            for n, a, b in zip(("dq_norm", "dk_norm"), dn, wn):
                close(n, a, b.grad, cfg["dtype"])
    if lead or tail:
        assert torch.all(layer.y[0, :lead] == 0) and torch.all(layer.y[0, T - prefix - tail:] == 0)
    return layer, cfg, host


F32 = dict(dtype="f32", d_model=64, nheads=2, d_head=32, E=4, k=2, causal=1)
BF = dict(dtype="bf16", d_model=256, nheads=4, d_head=64, E=5, k=3, causal=1)
W47 = dict(dtype="bf16", d_model=412, nheads=2, d_head=76, E=5, k=3, causal=1)


@pytest.mark.parametrize("base", [F32, BF, W47, dict(F32, d_head=33), dict(BF, causal=0)], ids=["f32", "bf16", "47m", "odd", "full"])
@pytest.mark.parametrize("norm,rope", [(False, 0), (True, 0), (False, 1), (True, 1)])
def test_packed_layer_forward_and_gradients(base, norm, rope):
    run(dict(base, rope=rope), [70, 1, 33, 128, 5], norm=norm)


@pytest.mark.parametrize("base", [F32, BF], ids=["f32", "bf16"])
def test_rows_of_no_sequence(base):
    """A padded batch: rows in front and behind are zeros in y and dx and give the weights nothing."""
    layer, cfg, _ = run(dict(base, rope=1), [40, 0, 17], norm=True, lead=7, tail=30)
    assert torch.all(layer.dx[0, :7] == 0) and torch.all(layer.dx[0, 64:] == 0)


@pytest.mark.parametrize("base", [F32, BF, W47], ids=["f32", "bf16", "47m"])
@pytest.mark.parametrize("lens", [[1] * 9, [20, 3, 64]])
@pytest.mark.parametrize("norm,rope", [(False, 0), (True, 1)])
def test_shared_prefix(base, lens, norm, rope):
    run(dict(base, rope=rope), lens, prefix=130, norm=norm, backward=False)


def test_shared_selection():
    run(dict(BF, rope=1), [70, 33], norm=True, shared=True)


def test_one_sequence_is_the_plain_layer():
    """fp32, no norms: one packed sequence of all rows gives the plain layer's results (another attention kernel: not to the last bit)."""
    layer, cfg, host = run(dict(F32, rope=1), [150])
    plain = DeviceLayer(dict(cfg), host)
    plain.forward()
    plain.backward()
    torch.cuda.synchronize()
    close("y", layer.y, plain.y.double().cpu(), "f32")
    for n in NAMES:
        close("d" + n, layer.dW[n], plain.dW[n].double().cpu(), "f32")


def test_routing_of_a_packed_call_is_that_of_its_rows():
    layer, cfg, host = run(dict(BF), [70, 33], backward=False)
    plain = DeviceLayer(dict(cfg), host)
    plain.forward()
    packing = binding.make_packing(torch.tensor([0, 70, 103], dtype=torch.int32, device="cuda"), 70)
    layer.ws = torch.empty(binding.switchhead_packed_workspace_bytes(layer.shape, packing), dtype=torch.uint8, device="cuda")
    W = layer.W
    binding.switchhead_forward_packed(layer.shape, packing, layer.x, W["W_Q"], W["W_K"], W["W_V"], W["W_O"], W["W_S"], W["W_D"], None, None, layer.y, layer.ws)
    a, b = layer.routing(), plain.routing()
    assert all(np.array_equal(a[n], b[n]) for n in ("idx", "perm", "offsets"))
