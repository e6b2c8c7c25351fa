"""The layer over packed sequences at the edges of what its description allows, on the GPU, against the float64 form and the bars of test_gpu_packed_layer."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import switchhead_oracle as orc
from paper_2312_07987_amd import binding
from paper_2312_07987_amd.inputs import make_inputs
from paper_2312_07987_amd.runner import DeviceLayer
from test_gpu_packed_layer import BAR, BF, F32, NAMES, close, reference

pytestmark = pytest.mark.gpu


class PackedCall:
    """A layer, its packing and its workspace on the GPU; forward() and backward() are the calls."""

    def __init__(self, cfg, offsets, rows, norm, eps, host=None, seed=3, dense=False, max_len=None):
        self.cfg = dict(cfg, B=1, T=rows)
        self.host = make_inputs(self.cfg, seed=seed) if host is None else host
        self.layer = DeviceLayer(self.cfg, self.host, dense=dense)
        d = cfg["d_head"]
        g = torch.Generator().manual_seed(5)
        self.w = [(1 + 0.2 * torch.randn(d, generator=g)).to(self.layer.tdtype) for _ in range(2)] if norm else None
        self.offsets = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        self.packing = binding.make_packing(self.offsets, rows if max_len is None else max_len, *([v.cuda() for v in self.w] if norm else (None, None)), norm_eps=eps)
        self.ws = torch.full((binding.switchhead_packed_workspace_bytes(self.layer.shape, self.packing),), 255, dtype=torch.uint8, device="cuda")
        self.dn = [torch.empty(d, device="cuda") if norm else None for _ in range(2)]

    def forward(self):
        l, W = self.layer, self.layer.W
        binding.switchhead_forward_packed(l.shape, self.packing, l.x, W["W_Q"], W["W_K"], W["W_V"], W["W_O"], W["W_S"], W["W_D"], l.b_S, l.b_D, l.y, self.ws)

    def backward(self):
        l, W, dW = self.layer, self.layer.W, self.layer.dW
        binding.switchhead_backward_packed(l.shape, self.packing, l.x, W["W_Q"], W["W_K"], W["W_V"], W["W_O"], W["W_S"], W["W_D"], l.dy, self.ws, l.dx,
                                           dW["W_Q"], dW["W_K"], dW["W_V"], dW["W_O"], dW["W_S"], dW["W_D"], l.db_S, l.db_D, *self.dn)

    def results(self):
        torch.cuda.synchronize()
        l = self.layer
        out = dict(y=l.y, dx=l.dx, **{"d" + n: l.dW[n] for n in NAMES})
        return {n: t for n, t in dict(out, dq_norm=self.dn[0], dk_norm=self.dn[1]).items() if t is not None}


@pytest.mark.parametrize("base", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("rope", [0, 1])
def test_padding_of_zeros_without_epsilon(base, rope):
    """norm_eps 0 and padding rows of zeros, whose norm has no value: they give nothing all the same."""
    cfg = dict(base, rope=rope)
    rows, lead, lens = 100, 9, [40, 17]
    at = slice(lead, lead + sum(lens))
    host = make_inputs(dict(cfg, B=1, T=rows), seed=3)
    for n in ("x", "dy"):
        kept = host[n][:, at].copy()
        host[n][:] = 0
        host[n][:, at] = kept
    p = PackedCall(cfg, [lead, lead + 40, lead + 57], rows, True, 0.0, host)
    p.forward()
    p.backward()
    got = p.results()
    t = {n: None if host.get(n) is None else torch.from_numpy(host[n][:, at] if n == "x" else host[n]).double().requires_grad_(True) for n in ("x",) + NAMES}
    wn = [v.double().requires_grad_(True) for v in p.w]
    y = reference(cfg, t, [0, 40, 57], 0, wn, 0.0)
    y.backward(torch.from_numpy(host["dy"][0, at]).double())
    for n in ("y", "dx"):
        out = torch.ones(rows, dtype=torch.bool)
        out[at] = False
        assert torch.all(got[n][0][out.cuda()] == 0), n
    close("y", got["y"][0, at], y, cfg["dtype"])
    close("dx", got["dx"][:, at], t["x"].grad, cfg["dtype"])
    for n in NAMES:
        close("d" + n, got["d" + n], t[n].grad, cfg["dtype"])
    close("dq_norm", got["dq_norm"], wn[0].grad, cfg["dtype"])
    close("dk_norm", got["dk_norm"], wn[1].grad, cfg["dtype"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["experts for queries and keys", "one table for both sides", "dense", "biases"])
def test_kinds_of_layers(kind, dtype):
    """Every kind of the layer, packed, against the float64 oracle's plain layer called for one sequence after the other."""
    cfg = dict(dict(F32) if dtype == "f32" else dict(BF), rope=1)
    cfg.update({"experts for queries and keys": dict(qk_experts=1), "dense": dict(E=1, k=1), "biases": dict(bias0=0.5)}.get(kind, {}))
    dense, lens, rows = kind == "dense", [70, 1, 33], 110
    host = make_inputs(dict(cfg, B=1, T=rows), seed=11, shared_router=kind == "one table for both sides")
    p = PackedCall(cfg, [0, 70, 71, 104], rows, False, 0.0, host, dense=dense)
    p.forward()
    p.backward()
    got, sums, at = p.results(), {}, 0
    y, dx = [], []
    W = {n: None if dense and n in ("W_S", "W_D") else host[n] for n in NAMES}
    for n in lens:
        f = orc.forward(host["x"][:, at:at + n], *[W[m] for m in NAMES], host["b_S"], host["b_D"], k=cfg["k"], causal=True, rope=True, T_q=None)
        g = orc.backward(host["x"][:, at:at + n], *[W[m] for m in NAMES], f, host["dy"][:, at:at + n])
        y.append(torch.from_numpy(np.asarray(f["y"], dtype=np.float64)))
        dx.append(torch.from_numpy(np.asarray(g["dx"], dtype=np.float64)))
        for m in NAMES:
            if W[m] is not None:
                sums[m] = sums.get(m, 0) + np.asarray(g["d" + m], dtype=np.float64)
        at += n
    assert torch.all(got["y"][0, at:] == 0) and torch.all(got["dx"][0, at:] == 0)
    close("y", got["y"][:, :at], torch.cat(y, 1), dtype)
    close("dx", got["dx"][:, :at], torch.cat(dx, 1), dtype)
    for m in sums:
        close("d" + m, got["d" + m], torch.from_numpy(sums[m]), dtype)


@pytest.mark.parametrize("base", [F32, BF], ids=["f32", "bf16"])
def test_captured_and_replayed_with_other_lengths(base):
    """A captured training step reads the offsets from the device: replays follow them, with other work between them."""
    p = PackedCall(dict(base, rope=1), [0, 30, 90], 100, True, 1e-5)

    def step():
        p.forward()
        p.backward()

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for offsets in ([0, 30, 90], [0, 1, 100], [10, 10, 60], [0, 30, 90]):
        p.offsets.copy_(torch.tensor(offsets, dtype=torch.int32))
        for t in p.results().values():
            t.fill_(7.0)
        graph.replay()
        again = {n: t.clone() for n, t in p.results().items()}
        step()
        for n, t in p.results().items():
            close(n, again[n], t.double().cpu(), "f32")   # (weight gradients may be added with fp32 atomics: not to the last bit)


def leftover(host, cfg, f, at):
    """What a sequence of one token may leave in dW_Q and dW_K, whose exact part is 0: its probability is 1, O = V to the bit, and dS = <dO, V> - <dO, O> is the
    difference of two sums of the same d products in two orders, each within d 2^-23 |dO| |V| (2^-23: sums that cut instead of rounding).
    dO is the gated sum of W_O dy, gates at most 1; an element of dW_Q is x s dS K, of dW_K x s dS Q."""
    d, most = cfg["d_head"], 0.0
    x, dy = host["x"][0, at.start].astype(np.float64), host["dy"][0, at.start].astype(np.float64)
    for h in range(cfg["nheads"]):
        dO = sum(np.linalg.norm(w.astype(np.float64) @ dy) for w in host["W_O"][h])
        Q, K, V = (np.linalg.norm(np.asarray(f[n], dtype=np.float64).reshape(-1, cfg["nheads"], d)[0, h]) for n in ("Q", "K", "V"))
        most = max(most, np.abs(x).max() * d ** -0.5 * 2 * d * 2.0 ** -23 * dO * V * max(Q, K))
    return most


@pytest.mark.parametrize("base", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("offsets,max_len", [([0, 40, 60], 25), ([0, 0, 1, 1, 1], 60), ([59, 60, 60], 1), ([0, 60], 1000)])
def test_bounds_on_the_lengths_and_empty_sequences(base, offsets, max_len):
    """Rows past max_len are rows of no sequence; empty sequences and single rows."""
    cfg, rows = dict(base, rope=1), 60
    host = make_inputs(dict(cfg, B=1, T=rows), seed=12)
    p = PackedCall(cfg, offsets, rows, False, 0.0, host, max_len=max_len)
    p.forward()
    p.backward()
    got = p.results()
    want = dict(y=np.zeros((1, rows, cfg["d_model"])), dx=np.zeros((1, rows, cfg["d_model"])), **{"d" + n: np.zeros(host[n].shape) for n in NAMES})
    none, rest = torch.ones(rows, dtype=torch.bool), 0.0
    for a, b in zip(offsets[:-1], offsets[1:]):
        at = slice(a, min(b, a + max_len))
        if at.start == at.stop:
            continue
        none[at] = False
        f = orc.forward(host["x"][:, at], *[host[m] for m in NAMES], None, None, k=cfg["k"], causal=True, rope=True, T_q=None)
        g = orc.backward(host["x"][:, at], *[host[m] for m in NAMES], f, host["dy"][:, at])
        want["y"][:, at], want["dx"][:, at] = f["y"], g["dx"]
        for n in NAMES:
            want["d" + n] += g["d" + n]
        if at.stop - at.start == 1:
            rest += leftover(host, cfg, f, at)
    for n in ("y", "dx"):
        assert torch.all(got[n][0][none.cuda()] == 0), n
    for n, w in want.items():
        slack = rest if n in ("dW_Q", "dW_K") else 0.0
        err, most = float((got[n].double().cpu() - torch.from_numpy(w)).abs().max()), float(np.abs(w).max())
        print(n, err, most, slack, flush=True)
        assert err <= BAR[cfg["dtype"]] * most + slack, n
