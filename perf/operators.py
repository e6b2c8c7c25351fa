"""The attention operators that stand beside the layer, as cases that can be timed: attention over packed sequences with grouped
heads (training steps, prompts, single tokens over caches), attention of a batch whose sequences share a prefix, and the norms of
queries and keys with the position rotation in the same pass.

`own` chooses between the plain form (elementary torch operations in 32 bits, angles in 64) and the package's operators.

A case is a dict.  Attention ("attention", "prefix"): `call` "train" (forward, then backward) or "forward"; `heads`, `kv_heads`,
`d_head`, `dtype`; `queries` and `keys`, the lengths of the sequences as texts; `prefix`, rows that all sequences share in front of their
own keys; `layout` "rows" (tensors of their own), "fused" (Q, K, V are views of one projection's output) or "cache" (keys and
values lie in rows of a cache of one length for all sequences).  Norms ("norm_rope"): `call` "train" or "forward", `tokens`, `heads`,
`kv_heads`, `d_head`, `rope_dim`, `far` (largest position), `dtype`, `layout` "rows" or "fused".
"""
import math
import random

import torch

own = False

EPS = 1e-6
THETA = 10000.0


# ----------------------------------------------------------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------------------------------------------------------
def _text(lengths):
    return " ".join(str(int(n)) for n in lengths)


def _lengths(text):
    return [int(n) for n in text.split()]


def _ragged(rng, n, low, high):
    """n lengths between low and high, spread over their logarithm."""
    return [min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))) for _ in range(n)]


def _attention(op, call, heads, kv_heads, d_head, dtype, queries, keys=None, prefix=0, layout="rows"):
    return dict(op=op, call=call, heads=heads, kv_heads=kv_heads, d_head=d_head, dtype=dtype, queries=_text(queries),
                keys=_text(queries if keys is None else keys), prefix=prefix, layout=layout)


def _norm(call, tokens, heads, kv_heads, d_head, rope_dim, far, dtype, layout="rows"):
    return dict(op="norm_rope", call=call, tokens=tokens, heads=heads, kv_heads=kv_heads, d_head=d_head, rope_dim=rope_dim, far=far,
                dtype=dtype, layout=layout)


def listed():
    rng = random.Random(7)
    named = {
        # a unit test or a toy model in fp32: the package's smallest workload as two packed sequences; launches and latency
        "toy_f32_train": _attention("attention", "train", 2, 2, 32, "f32", [64, 64]),
        # training the 47M model on documents of at most its context length (head width 76: rows of 8-byte alignment)
        "packed_47m_train": _attention("attention", "train", 2, 2, 76, "bf16", _ragged(rng, 96, 20, 256)),
        # training the 262M model's layer on documents of very different lengths
        "packed_262m_train": _attention("attention", "train", 4, 4, 128, "bf16", [4096, 17, 1, 2048, 655, 3001, 129, 1500, 64, 2500, 333, 1024]),
        # the dense layer's twenty heads of 80 in groups of five, two long sequences and a single token, views of one projection
        "grouped_train": _attention("attention", "train", 20, 4, 80, "bf16", [4096, 1, 2500], layout="fused"),
        # a long prompt of a grouped-head model before its first token
        "long_prompt": _attention("attention", "forward", 32, 8, 128, "bf16", [8192]),
        # the second half of prompts that arrive in pieces: queries behind keys that are there already
        "prompt_pieces": _attention("attention", "forward", 4, 4, 128, "bf16", [512, 300, 64], [2500, 300, 4000]),
        # a token for each of a few users over caches of the 262M layer's heads
        "decode": _attention("attention", "forward", 4, 4, 128, "bf16", [1] * 16, _ragged(rng, 16, 500, 4000), layout="cache"),
        # a token for each of many users, grouped heads, long caches: bandwidth
        "decode_grouped": _attention("attention", "forward", 32, 8, 128, "bf16", [1] * 32, _ragged(rng, 32, 2000, 32768), layout="cache"),
        # a token for each of many users behind one system prompt
        "prefix_decode": _attention("prefix", "forward", 32, 8, 128, "bf16", [1] * 64, _ragged(rng, 64, 1, 500), 4096),
        # questions of different lengths about one document
        "prefix_questions": _attention("prefix", "forward", 4, 4, 128, "bf16", _ragged(rng, 12, 10, 400), None, 2048),
        # a training step's queries and keys of a grouped-head model, views of one projection
        "norm_rope_train": _norm("train", 16384, 32, 8, 128, 128, 4096, "bf16", "fused"),
        # a decoding step of the 262M layer's heads, far into long texts: launch and latency
        "norm_rope_decode": _norm("forward", 64, 4, 4, 128, 128, 200000, "bf16"),
    }
    return [dict(case, name=name) for name, case in named.items()]


# a drawn case stays below the largest listed ones: multiply-adds of attention, elements of the norms, plain scores in memory
MAX_FLOPS = 4e11
MAX_BYTES = 2.0e9
MAX_SCORES = 2.2e9
MAX_ELEMENTS = 16384 * 40 * 128


def _log(rng, low, high):
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    while True:
        kind = rng.choice(["train", "train", "prompt", "decode", "decode", "prefix", "prefix", "norm", "norm"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        kv_heads = rng.choice([1, 2, 2, 4, 4, 8])
        heads = kv_heads * rng.choice([1, 1, 2, 4, 5, 8])
        if kind == "norm":
            d_head = rng.choice([32, 48, 64, 76, 80, 100, 128, 128, 256])
            rope_dim = rng.choice([d_head, d_head, d_head // 4 * 2, 0])
            case = _norm(rng.choice(["train", "forward"]), _log(rng, 1, 16384), heads, kv_heads, d_head, rope_dim,
                         _log(rng, 100, 1000000), dtype, rng.choice(["rows", "fused"]))
            if case["tokens"] * (heads + kv_heads) * d_head <= MAX_ELEMENTS:
                return case
            continue
        d_head = rng.choice([32, 48, 64, 64, 76, 80, 100, 128, 128, 128, 256])
        prefix, layout = 0, "rows"
        if kind == "train":
            queries = _ragged(rng, _log(rng, 1, 100), 1, rng.choice([128, 512, 2048, 4096]))
            keys, layout = queries, rng.choice(["rows", "fused"])
        elif kind == "prompt":
            queries = _ragged(rng, _log(rng, 1, 16), 1, rng.choice([512, 2048, 8192]))
            keys = [max(1, n + rng.choice([0, 0, _log(rng, 1, 4096), -(n // 3)])) for n in queries]   # (the last: first queries that see nothing)
        elif kind == "decode":
            queries = [rng.choice([1, 1, 1, 2, 5])] * _log(rng, 1, 64)
            keys = [max(n, k) for n, k in zip(queries, _ragged(rng, len(queries), 1, rng.choice([500, 4000, 32768])))]
            layout = rng.choice(["rows", "cache", "cache"])
        else:
            prefix = _log(rng, 50, 8192)
            n = _log(rng, 1, 64)
            queries = [1] * n if rng.random() < 0.6 else _ragged(rng, n, 1, 300)
            keys = [k + rng.choice([0, _log(rng, 1, 500)]) for k in queries]
        case = _attention("prefix" if prefix else "attention", "train" if kind == "train" else "forward", heads, kv_heads, d_head,
                          dtype, queries, keys, prefix, layout)
        cost = work(case)
        scores = len(queries) * heads * max(queries) * (max(keys) + prefix)
        room = len(queries) * max(keys) * kv_heads * d_head * 8
        limit = MAX_FLOPS / 12 if dtype == "f32" else MAX_FLOPS
        if cost["flops"] <= limit and cost["bytes"] <= MAX_BYTES and scores <= MAX_SCORES and room <= 9e9:
            return case


def _element(case):
    return 4 if case["dtype"] == "f32" else 2


def _pairs(queries, keys, prefix):
    """Visible (query, key) pairs of one head under the causal mask."""
    total = 0
    for n, k in zip(queries, keys):
        total += n * prefix
        # query i sees k - n + i + 1 own keys, none where that is negative
        first = max(0, n - k)
        total += (n - first) * (k - n + first + 1 + k) // 2 if n > first else 0
    return total


def work(case):
    if case["op"] == "norm_rope":
        elements = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["d_head"]
        train = case["call"] == "train"
        # train: x and dy read, y and dx written; forward: x read, y written
        return {"bytes": elements * _element(case) * (4 if train else 2) + case["tokens"] * 4, "flops": elements * (24 if train else 10)}
    queries, keys = _lengths(case["queries"]), _lengths(case["keys"])
    pairs = _pairs(queries, keys, case["prefix"]) * case["heads"]
    q = sum(queries) * case["heads"] * case["d_head"] * _element(case)
    kv = (sum(keys) + case["prefix"]) * case["kv_heads"] * case["d_head"] * _element(case)
    if case["call"] == "train":
        # Q, K, V, dO read; O, lse, dQ, dK, dV written
        return {"bytes": 4 * q + 4 * kv + sum(queries) * case["heads"] * 4, "flops": 14 * case["d_head"] * pairs}
    return {"bytes": 2 * q + 2 * kv, "flops": 4 * case["d_head"] * pairs}


# ----------------------------------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _rows(gen, case, rows, heads, scale=1.0):
    # (a sequence count of zero tokens still needs memory to point at)
    t = torch.randn((max(rows, 1), heads, case["d_head"]), generator=gen, device="cuda", dtype=torch.float32)
    return (t * scale).to(_dtype(case))


def _offsets(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    heads, kv_heads, d = case["heads"], case["kv_heads"], case["d_head"]
    state = dict(case=case)
    if case["op"] == "norm_rope":
        n = case["tokens"]
        # the rows of a projection have different sizes from token to token and head to head
        size = torch.exp(torch.randn((n, heads + kv_heads, 1), generator=gen, device="cuda") * 0.5)
        x = (torch.randn((n, heads + kv_heads, d), generator=gen, device="cuda") * size).to(_dtype(case))
        if case["layout"] == "fused":
            # one projection's output: query heads, key heads, and the value heads that stay as they are
            qkv = torch.empty((n, heads + 2 * kv_heads, d), device="cuda", dtype=_dtype(case))
            qkv[:, :heads + kv_heads] = x
            qkv[:, heads + kv_heads:] = 1
            state.update(Q=qkv[:, :heads], K=qkv[:, heads:heads + kv_heads])
        else:
            state.update(Q=x[:, :heads].contiguous(), K=x[:, heads:].contiguous())
        state["w_Q"] = (1 + 0.1 * torch.randn((d,), generator=gen, device="cuda")).to(_dtype(case))
        state["w_K"] = (1 + 0.1 * torch.randn((d,), generator=gen, device="cuda")).to(_dtype(case))
        # documents that begin anywhere: positions count up and start again
        start = torch.randint(0, case["far"], (1,), generator=gen, device="cuda")
        state["positions"] = ((torch.arange(n, device="cuda") + start) % (case["far"] + 1)).to(torch.int32)
        if case["call"] == "train":
            state["dY_Q"] = _rows(gen, case, n, heads)
            state["dY_K"] = _rows(gen, case, n, kv_heads)
        return state
    queries, keys = _lengths(case["queries"]), _lengths(case["keys"])
    state.update(max_q=max(queries), max_k=max(keys), q_offsets=_offsets(queries))
    rows_q = sum(queries)
    if case["layout"] == "fused":
        qkv = _rows(gen, case, rows_q, heads + 2 * kv_heads)
        state.update(Q=qkv[:, :heads], K=qkv[:, heads:heads + kv_heads], V=qkv[:, heads + kv_heads:], k_offsets=state["q_offsets"])
    elif case["layout"] == "cache":
        # a place of one length for every sequence, partly filled; what lies behind a sequence's keys is left from others
        room = -(-max(keys) // 64) * 64
        state.update(Q=_rows(gen, case, rows_q, heads), K=_rows(gen, case, room * len(keys), kv_heads), V=_rows(gen, case, room * len(keys), kv_heads),
                     k_offsets=_offsets([room] * len(keys)), k_lengths=torch.tensor(keys, dtype=torch.int32, device="cuda"))
    else:
        state.update(Q=_rows(gen, case, rows_q, heads), K=_rows(gen, case, sum(keys), kv_heads), V=_rows(gen, case, sum(keys), kv_heads),
                     k_offsets=_offsets(keys))
    if case["prefix"]:
        state.update(K_prefix=_rows(gen, case, case["prefix"], kv_heads), V_prefix=_rows(gen, case, case["prefix"], kv_heads))
    if case["call"] == "train":
        state["dO"] = _rows(gen, case, rows_q, heads)
    return state


# ----------------------------------------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------------------------------------
def run(state):
    if own:
        return _own_norm(state) if state["case"]["op"] == "norm_rope" else _own_attention(state)
    return _plain_norm(state) if state["case"]["op"] == "norm_rope" else _plain_attention(state)


def _plain_rotation(positions, rope_dim, d, sign):
    """cos and sin of every pair of every token, [tokens, 1, d / 2]; pairs that are not turned have angle 0."""
    pair = torch.arange(d // 2, device=positions.device, dtype=torch.float64)
    rate = torch.where(2 * pair < rope_dim, torch.pow(THETA, -2.0 * pair / max(rope_dim, 1)), 0.0)
    angle = positions.to(torch.float64)[:, None, None] * rate
    return torch.cos(angle).float(), sign * torch.sin(angle).float()


def _turn(x, cos, sin):
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * cos - b * sin, a * sin + b * cos), -1).reshape(x.shape)


def _plain_norm_rows(x, w, positions, rope_dim, dY):
    x32, w32 = x.float(), w.float()
    r = 1.0 / torch.sqrt((x32 * x32).mean(-1, keepdim=True) + EPS)
    u = x32 * r
    cos, sin = _plain_rotation(positions, rope_dim, x.shape[-1], 1.0)
    y = _turn(u * w32, cos, sin).to(x.dtype)
    if dY is None:
        return y, None, None
    dn = _turn(dY.float(), cos, -sin)
    g = dn * w32
    dx = r * (g - u * (g * u).mean(-1, keepdim=True))
    return y, dx.to(x.dtype), (dn * u).sum((0, 1))


def _plain_norm(state):
    rope_dim, train = state["case"]["rope_dim"], state["case"]["call"] == "train"
    y_q, d_q, dw_q = _plain_norm_rows(state["Q"], state["w_Q"], state["positions"], rope_dim, state["dY_Q"] if train else None)
    y_k, d_k, dw_k = _plain_norm_rows(state["K"], state["w_K"], state["positions"], rope_dim, state["dY_K"] if train else None)
    if train:
        return dict(Y_Q=y_q, Y_K=y_k, dQ=d_q, dK=d_k, dw_Q=dw_q, dw_K=dw_k)
    return dict(Y_Q=y_q, Y_K=y_k)


def _padded(x, offsets, lengths, most):
    """[sequences, most, heads, d] in 32 bits, zeros behind a sequence's rows; the rows' validity."""
    at = torch.arange(most, device=x.device)
    valid = at < lengths[:, None]
    rows = (offsets[:-1, None] + at).clamp(max=x.shape[0] - 1)
    return x[rows].float() * valid[..., None, None], valid


def _places(offsets, rows):
    """Sequence and position of every packed row."""
    at = torch.arange(rows, device=offsets.device, dtype=offsets.dtype)
    seq = (torch.searchsorted(offsets, at, right=True) - 1).clamp(0, offsets.numel() - 2)
    return seq, (at - offsets[seq]).long()


def _plain_attention(state):
    case = state["case"]
    Q, K, V = state["Q"], state["K"], state["V"]
    kv_heads, d = case["kv_heads"], case["d_head"]
    group = case["heads"] // kv_heads
    scale = 1.0 / math.sqrt(d)
    q_off, k_off = state["q_offsets"].long(), state["k_offsets"].long()
    q_len = q_off[1:] - q_off[:-1]
    k_len = state["k_lengths"].long() if "k_lengths" in state else k_off[1:] - k_off[:-1]
    max_q, max_k = state["max_q"], state["max_k"]
    n = q_len.numel()

    def by_group(x):   # [n, max_q, heads, d] -> [n, kv_heads, max_q * group, d]
        return x.reshape(n, max_q, kv_heads, group, -1).permute(0, 2, 1, 3, 4).reshape(n, kv_heads, max_q * group, -1)

    def to_rows(x, width):   # and back, to packed rows
        x = x.reshape(n, kv_heads, max_q, group, width).permute(0, 2, 1, 3, 4).reshape(n, max_q, kv_heads * group, width)
        seq, at = _places(q_off, Q.shape[0])
        return x[seq, at]

    q, _ = _padded(Q, q_off, q_len, max_q)
    k, k_valid = _padded(K, k_off, k_len, max_k)
    v, _ = _padded(V, k_off, k_len, max_k)
    q = by_group(q)
    k, v = k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous()   # [n, kv_heads, max_k, d]
    at_q = torch.arange(max_q, device=Q.device).repeat_interleave(group)
    at_k = torch.arange(max_k, device=Q.device)
    visible = k_valid[:, None, :] & (at_k <= (k_len - q_len)[:, None, None] + at_q[:, None])   # [n, max_q * group, max_k]
    prefix = case["prefix"]
    if prefix:
        kp, vp = state["K_prefix"].float().transpose(0, 1), state["V_prefix"].float().transpose(0, 1)   # [kv_heads, prefix, d]
        k = torch.cat((kp.expand(n, -1, -1, -1), k), 2)
        v = torch.cat((vp.expand(n, -1, -1, -1), v), 2)
        visible = torch.cat((visible.new_ones((n, max_q * group, prefix)), visible), 2)
    visible = visible[:, None]
    s = (torch.matmul(q, k.transpose(2, 3).contiguous()) * scale).masked_fill_(~visible, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp_(s.sub_(torch.where(torch.isfinite(m), m, 0.0)))   # a row that sees nothing: zeros
    total = p.sum(-1, keepdim=True)
    lse = m + torch.log(total)
    p.div_(torch.where(total > 0, total, 1.0))
    o = torch.matmul(p, v)
    O = to_rows(o, d).to(Q.dtype)
    if case["call"] != "train":
        return dict(O=O)
    dO, _ = _padded(state["dO"], q_off, q_len, max_q)
    dO = by_group(dO)
    ds = torch.matmul(dO, v.transpose(2, 3).contiguous()).sub_((dO * o).sum(-1, keepdim=True)).mul_(p)
    dV = torch.matmul(p.transpose(2, 3).contiguous(), dO)
    dQ = torch.matmul(ds, k) * scale
    dK = torch.matmul(ds.transpose(2, 3).contiguous(), q) * scale
    seq, at = _places(k_off, K.shape[0])
    return dict(O=O, lse=to_rows(lse, 1)[..., 0].t().contiguous(), dQ=to_rows(dQ, d).to(Q.dtype),
                dK=dK.transpose(1, 2)[seq, at].to(K.dtype), dV=dV.transpose(1, 2)[seq, at].to(V.dtype))


def _own_norm(state):
    from paper_2312_07987_amd import binding
    Q, K, train = state["Q"], state["K"], state["case"]["call"] == "train"
    kept = state.get("kept")
    if kept is None:   # what a program keeps from step to step: the output buffers and the workspace
        Y_Q, Y_K = torch.empty(Q.shape, dtype=Q.dtype, device=Q.device), torch.empty(K.shape, dtype=K.dtype, device=K.device)
        plan = binding.make_qk_norm(Q, K, Y_Q, Y_K, rope_dim=state["case"]["rope_dim"], eps=EPS, theta=THETA)
        kept = state["kept"] = dict(Y_Q=Y_Q, Y_K=Y_K, plan=plan)
        if train:
            # gradients lie as their tensors do
            base = torch.empty_strided((Q.shape[0], Q.stride(0) // Q.stride(1), Q.shape[2]), (Q.stride(0), Q.stride(1), 1), dtype=Q.dtype, device=Q.device)
            fused = state["case"]["layout"] == "fused"
            heads = Q.shape[1]
            kept["dQ"] = base[:, :heads]
            kept["dK"] = base[:, heads:heads + K.shape[1]] if fused else torch.empty_like(K)
            kept["dw_Q"], kept["dw_K"] = (torch.empty(Q.shape[2], dtype=torch.float32, device=Q.device) for _ in range(2))
            kept["ws"] = torch.empty(binding.switchhead_qk_norm_workspace_bytes(plan), dtype=torch.uint8, device=Q.device)
    binding.switchhead_qk_norm_rope_forward(kept["plan"], Q, K, state["w_Q"], state["w_K"], state["positions"], kept["Y_Q"], kept["Y_K"])
    if not train:
        return dict(Y_Q=kept["Y_Q"], Y_K=kept["Y_K"])
    binding.switchhead_qk_norm_rope_backward(kept["plan"], Q, K, state["w_Q"], state["w_K"], state["positions"], state["dY_Q"], state["dY_K"],
                                             kept["dQ"], kept["dK"], kept["dw_Q"], kept["dw_K"], kept["ws"])
    return {n: kept[n] for n in ("Y_Q", "Y_K", "dQ", "dK", "dw_Q", "dw_K")}


def _own_attention(state):
    from paper_2312_07987_amd import binding
    Q, K, V, train = state["Q"], state["K"], state["V"], state["case"]["call"] == "train"
    prefix = dict(K_prefix=state.get("K_prefix"), V_prefix=state.get("V_prefix"))
    kept = state.get("kept")
    if kept is None:   # what a program keeps from step to step: the output buffers and the workspace
        O = torch.empty(Q.shape, dtype=Q.dtype, device=Q.device)
        plan = binding.make_attention(Q, K, V, O, nseq=state["q_offsets"].numel() - 1, max_q=state["max_q"], max_k=state["max_k"], causal=1, **prefix)
        kept = state["kept"] = dict(O=O, plan=plan, lse=None)
        kept["ws"] = torch.empty(binding.switchhead_attention_workspace_bytes(plan, backward=train), dtype=torch.uint8, device=Q.device)
        if train:
            kept["lse"] = torch.empty((Q.shape[1], Q.shape[0]), dtype=torch.float32, device=Q.device)
            if state["case"]["layout"] == "fused":   # gradients lie as their tensors do
                heads, kv = Q.shape[1], K.shape[1]
                dqkv = torch.empty((Q.shape[0], heads + 2 * kv, Q.shape[2]), dtype=Q.dtype, device=Q.device)
                kept.update(dQ=dqkv[:, :heads], dK=dqkv[:, heads:heads + kv], dV=dqkv[:, heads + kv:])
            else:
                kept.update(dQ=torch.empty_like(Q), dK=torch.empty_like(K), dV=torch.empty_like(V))
    q_off, k_off, k_len = state["q_offsets"], state["k_offsets"], state.get("k_lengths")
    binding.switchhead_attention_forward(kept["plan"], Q, K, V, q_off, k_off, kept["O"], kept["lse"], kept["ws"], k_lengths=k_len, **prefix)
    if not train:
        return dict(O=kept["O"])
    binding.switchhead_attention_backward(kept["plan"], Q, K, V, kept["O"], state["dO"], kept["lse"], q_off, k_off, kept["dQ"], kept["dK"], kept["dV"],
                                          kept["ws"], k_lengths=k_len)
    return {n: kept[n] for n in ("O", "lse", "dQ", "dK", "dV")}


# ----------------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits: one sequence and one head (or one tensor's rows as complex numbers) at a time
# ----------------------------------------------------------------------------------------------------------------------------
def _exact_norm_rows(x, w, positions, rope_dim, dY):
    x, w = x.double(), w.double()
    half = rope_dim // 2
    size = torch.linalg.vector_norm(x, dim=-1, keepdim=True) / math.sqrt(x.shape[-1])
    r = (size ** 2 + EPS) ** -0.5
    rates = torch.tensor([THETA ** (-2.0 * i / rope_dim) for i in range(half)], dtype=torch.float64, device=x.device)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), positions.double()[:, None] * rates)[:, None]   # [tokens, 1, half]

    def turned(t, by):
        if not half:
            return t
        z = torch.view_as_complex(t[..., :rope_dim].reshape(*t.shape[:-1], half, 2).contiguous()) * by
        return torch.cat((torch.view_as_real(z).flatten(-2), t[..., rope_dim:]), -1)

    y = turned(x * r * w, turn)
    if dY is None:
        return y, None, None
    dn = turned(dY.double(), turn.conj())
    dw = torch.einsum("nhd,nhd->d", dn, x * r)
    g = dn * w
    dx = g * r - x * r ** 3 * (g * x).mean(-1, keepdim=True)
    return y, dx, dw


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "norm_rope":
        train = case["call"] == "train"
        y_q, d_q, dw_q = _exact_norm_rows(state["Q"], state["w_Q"], state["positions"], case["rope_dim"], state["dY_Q"] if train else None)
        y_k, d_k, dw_k = _exact_norm_rows(state["K"], state["w_K"], state["positions"], case["rope_dim"], state["dY_K"] if train else None)
        return dict(Y_Q=y_q, Y_K=y_k, dQ=d_q, dK=d_k, dw_Q=dw_q, dw_K=dw_k) if train else dict(Y_Q=y_q, Y_K=y_k)
    Q, K, V = state["Q"], state["K"], state["V"]
    heads, group, d = case["heads"], case["heads"] // case["kv_heads"], case["d_head"]
    queries, keys = _lengths(case["queries"]), _lengths(case["keys"])
    train = case["call"] == "train"
    wide = dict(dtype=torch.float64, device=Q.device)
    O, lse = torch.zeros(Q.shape, **wide), torch.full((heads, Q.shape[0]), -math.inf, **wide)
    dQ, dK, dV = (torch.zeros(t.shape, **wide) for t in (Q, K, V)) if train else (None, None, None)
    k_begin = state["k_offsets"].tolist()
    q0 = 0
    for i, (n, k) in enumerate(zip(queries, keys)):
        q_rows, k_rows = slice(q0, q0 + n), slice(k_begin[i], k_begin[i] + k)
        q0 += n
        hidden = torch.ones((n, k), dtype=torch.bool, device=Q.device).triu(k - n + 1)
        for h in range(heads):
            q, kk, v = Q[q_rows, h].double(), K[k_rows, h // group].double(), V[k_rows, h // group].double()
            s = (q @ kk.t() / math.sqrt(d)).masked_fill_(hidden, -math.inf)
            if case["prefix"]:
                s = torch.cat((q @ state["K_prefix"][:, h // group].double().t() / math.sqrt(d), s), 1)
                v = torch.cat((state["V_prefix"][:, h // group].double(), v), 0)
            row = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(torch.isfinite(row), row, 0.0)[:, None])
            O[q_rows, h] = p @ v
            lse[h, q_rows] = row
            if train:
                g = state["dO"][q_rows, h].double()
                dp = g @ v.t()
                ds = p * (dp - (p * dp).sum(1, keepdim=True))
                dQ[q_rows, h] = ds @ kk / math.sqrt(d)
                dK[k_rows, h // group] += ds.t() @ q / math.sqrt(d)
                dV[k_rows, h // group] += p.t() @ g
    return dict(O=O, lse=lse, dQ=dQ, dK=dK, dV=dV) if train else dict(O=O)
