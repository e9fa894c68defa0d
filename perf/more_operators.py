"""The operators that carry a GRPO update through the layers of the model, as timed cases.

Scoring and loss give a gradient at the logits; the way back to the weights leads through attention and the norms of
the residual stream, and ends in the optimiser's step.  The cases are packed attention with the log-sum-exp that its
gradient needs, that gradient, the root-mean-square norm behind a residual addition (with an output in bf16 or in 8
bits) and its gradient, and an AdamW step over all tensors of a layer or a model, from the tiny fp32 model of the smoke
test to the widths of the 7B, 14B and 72B decoders.

Each operator has a plain form (``own`` false): elementary torch operations in 32 bits.  ``exact`` is the definition in
64 bits.  Eight-bit numbers are e4m3 with a power of two as scale: one for a row of the norm's output, one for 128
elements of an optimiser state, which is rounded up or down by the bits of a counter hash.
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2, "e4m3": 1}
INF = float("inf")
E4M3 = torch.float8_e4m3fn
BLOCK = 128


def listed():
    return [
        # the tiny fp32 model: eight sequences of a prompt and its completion, where only latency counts
        {"name": "attention_tiny", "kind": "attention", "heads": 4, "kv": 4, "hd": 32, "seqs": 8, "shortest": 17, "longest": 32, "queries": 0, "dtype": "fp32", "room": 0, "causal": True},
        # the 7B benchmark's completions (prompt 256, up to 512 new tokens) packed for scoring
        {"name": "attention_update_7b", "kind": "attention", "heads": 28, "kv": 4, "hd": 128, "seqs": 16, "shortest": 257, "longest": 768, "queries": 0, "dtype": "bf16", "room": 0, "causal": True},
        # the next token of 16 sequences over keys of unequal number: few rows, long axis
        {"name": "attention_one_token_72b", "kind": "attention", "heads": 64, "kv": 8, "hd": 128, "seqs": 16, "shortest": 1024, "longest": 8192, "queries": 1, "dtype": "bf16", "room": 0, "causal": True},
        # the gradient of the tiny fp32 model, sequences in places of equal size
        {"name": "attention_backward_tiny", "kind": "attention_backward", "heads": 4, "kv": 4, "hd": 32, "seqs": 8, "shortest": 17, "longest": 32, "queries": 0, "dtype": "fp32", "room": 8, "causal": True},
        # the gradient of the 7B benchmark's packed completions
        {"name": "attention_backward_7b", "kind": "attention_backward", "heads": 28, "kv": 4, "hd": 128, "seqs": 16, "shortest": 257, "longest": 768, "queries": 0, "dtype": "bf16", "room": 0, "causal": True},
        # one long completion at the 14B model's heads
        {"name": "attention_backward_long_14b", "kind": "attention_backward", "heads": 40, "kv": 8, "hd": 128, "seqs": 1, "shortest": 8192, "longest": 8192, "queries": 0, "dtype": "bf16", "room": 0, "causal": True},
        # a decode step's norm: the attention's output joins the fp32 residual stream of 64 rows
        {"name": "norm_decode_7b", "kind": "norm", "rows": 64, "dim": 3584, "x": "fp32", "delta": "bf16", "y": "bf16"},
        # a prefill's rows at the 72B model's width, for products of 8-bit operands
        {"name": "norm_8bit_72b", "kind": "norm", "rows": 16384, "dim": 8192, "x": "fp32", "delta": "bf16", "y": "e4m3"},
        # bf16 rows of an odd width
        {"name": "norm_backward_odd", "kind": "norm_backward", "rows": 259, "dim": 1003, "x": "bf16", "dy": "bf16", "dx": "bf16", "inner": True},
        # the gradient of a micro-batch of 16 completions of the 7B benchmark
        {"name": "norm_backward_7b", "kind": "norm_backward", "rows": 12288, "dim": 3584, "x": "fp32", "dy": "bf16", "dx": "fp32", "inner": True},
        # every tensor of the tiny model's layers, states in 32 bits
        {"name": "adamw_tiny", "kind": "adamw", "layers": 2, "d": 128, "kvd": 128, "ff": 512, "param": "fp32", "grad": "fp32", "state": "fp32", "copy": False},
        # a layer of the 7B model: fp32 weights with a bf16 copy for the next rollout, states in 8 bits
        {"name": "adamw_8bit_7b", "kind": "adamw", "layers": 1, "d": 3584, "kvd": 512, "ff": 18944, "param": "fp32", "grad": "bf16", "state": "e4m3", "copy": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention_backward", "attention_backward", "attention_backward", "norm",
                       "norm_backward", "adamw"])
    if kind.startswith("attention"):
        heads, kv, hd = rng.choice([(4, 4, 32), (28, 4, 128), (40, 8, 128), (64, 8, 128), (16, 16, 64), (14, 2, 64), (32, 8, 128)])
        dtype = rng.choice(["fp32", "bf16", "bf16", "bf16"])
        longest = _log(rng, 1, 8192 if dtype == "bf16" else 2048)
        # at most the pairs of the longest listed sequence, padded
        most = 8192 * 8192 * 40 // (longest * longest * heads)
        queries = rng.choice([0, 0, 0, 1, _log(rng, 1, longest)])
        if queries:
            queries = min(queries, longest)
        seqs = _log(rng, 1, max(1, min(64, most, 65536 // longest)))
        return {"kind": kind, "heads": heads, "kv": kv, "hd": hd, "seqs": seqs, "shortest": max(1, longest // rng.choice([1, 2, 8])),
                "longest": longest, "queries": queries, "dtype": dtype, "room": rng.choice([0, 0, 0, 5]), "causal": rng.random() < 0.8}
    if kind.startswith("norm"):
        dim = rng.choice([128, 544, 640, 1000, 3584, 5120, 8192, _log(rng, 16, 12000)])
        rows = _log(rng, 1, min(65536, 16384 * 8192 // dim // 2))
        case = {"kind": kind, "rows": rows, "dim": dim, "x": rng.choice(["fp32", "bf16"])}
        if kind == "norm":
            return {**case, "delta": rng.choice(["", "bf16", "bf16", "fp32"]), "y": rng.choice(["bf16", "bf16", "e4m3", "fp32"])}
        return {**case, "dy": rng.choice(["bf16", "bf16", "fp32"]), "dx": rng.choice(["bf16", "fp32"]), "inner": rng.random() < 0.7}
    param = rng.choice(["fp32", "fp32", "bf16"])
    # widths from an adapter's few hundred to about half a 7B layer, in as many layers
    d = _log(rng, 96, 2600)
    layer = 2 * d * d + 2 * d * (d // 4) + 3 * d * 4 * d
    return {"kind": kind, "layers": _log(rng, 1, max(1, min(28, 200_000_000 // layer))), "d": d, "kvd": d // 4, "ff": 4 * d, "param": param,
            "grad": rng.choice(["fp32", "bf16"]), "state": rng.choice(["fp32", "e4m3", "e4m3"]), "copy": param == "fp32" and rng.random() < 0.5}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 2 + 1)


def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    x = torch.randn(shape, generator=g, device=DEV, dtype=dtype)
    return x.mul_(scale) if scale != 1.0 else x


def _zeros(*shape, dtype=torch.float32):
    return torch.zeros(shape, device=DEV, dtype=dtype)


def _key_lengths(case):
    """Evenly spread from the shortest to the longest."""
    S, lo, hi = case["seqs"], case["shortest"], case["longest"]
    return [hi] if S == 1 else [lo + (hi - lo) * s // (S - 1) for s in range(S)]


def _query_lengths(case):
    return [min(case["queries"], n) if case["queries"] else n for n in _key_lengths(case)]


def _places(lengths, room):
    """First rows of the sequences, one behind the last, and the number of rows: packed, or with unused rows behind each."""
    starts, at = [], 0
    for n in lengths:
        starts.append(at)
        at += n + room
    return starts + [at], at


def _rows_index(starts, lengths):
    """Rows of a padded batch [sequences, longest] in the packed matrix, and which of them are there."""
    t = torch.arange(int(max(lengths)), device=DEV)
    s = torch.tensor(starts[:-1], device=DEV)
    n = torch.tensor(lengths, device=DEV)
    there = t[None] < n[:, None]
    return (s[:, None] + t[None]).masked_fill(~there, 0), there


def _adamw_sizes(case):
    d, kvd, ff = case["d"], case["kvd"], case["ff"]
    one = [d, d * d, kvd * d, kvd * d, d * d, d, ff * d, ff * d, d * ff]
    return one * case["layers"] + [d]


HYPER = {"lr": 3e-4, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "step": 7, "seed": 0x5EED0FADA}
DECAY = 0.1
SCALE_OF_SCORES = 1.25  # times the usual 1 / sqrt(head_dim)
EPS = 1e-6


def _mask64(x):
    return x & 0xFFFFFFFFFFFFFFFF


def _mix64(x):
    x = _mask64((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9)
    x = _mask64((x ^ (x >> 27)) * 0x94D049BB133111EB)
    return x ^ (x >> 31)


def _tensor_key(tensor):
    """Key of a tensor's counter hash in a step (its first 2^32 elements')."""
    gold = 0x9E3779B97F4A7C15
    s = _mix64(_mask64(HYPER["seed"] + gold * HYPER["step"]))
    return _mix64(_mask64(s + gold * (tensor + 1)))


def prepare(case, seed):
    g = _gen(seed)
    st = {"case": case}
    kind = case["kind"]
    if kind.startswith("attention"):
        _prepare_attention(case, g, st)
    elif kind == "norm":
        n, d = case["rows"], case["dim"]
        st["x"] = _randn(g, n, d, dtype=TYPES[case["x"]], scale=3.0)
        st["delta"] = _randn(g, n, d, dtype=TYPES[case["delta"]]) if case["delta"] else None
        st["gain"] = 1.0 + _randn(g, d, scale=0.1)
        st["h"] = _zeros(n, d, dtype=TYPES[case["x"]]) if case["delta"] else None
        st["y"] = _zeros(n, d, dtype=E4M3 if case["y"] == "e4m3" else TYPES[case["y"]])
        st["scales"] = _zeros(n) if case["y"] == "e4m3" else None
        st["rstd"] = _zeros(n)
    elif kind == "norm_backward":
        n, d = case["rows"], case["dim"]
        st["h"] = _randn(g, n, d, dtype=TYPES[case["x"]], scale=3.0)
        st["gain"] = 1.0 + _randn(g, d, scale=0.1)
        st["rstd"] = torch.rsqrt(st["h"].double().square().mean(1) + EPS).float()
        st["dy"] = _randn(g, n, d, dtype=TYPES[case["dy"]], scale=0.01)
        st["inner"] = _randn(g, n, d, dtype=TYPES[case["dx"]], scale=0.01) if case["inner"] else None
        st["dx"] = _zeros(n, d, dtype=TYPES[case["dx"]])
        st["dgain"] = _zeros(d)
        if own:
            import paper_2608_11226_amd as R

            st["bytes"] = R.rollout_rms_norm_backward_workspace(n, d)
            st["ws"] = _zeros(max(1, st["bytes"]), dtype=torch.uint8)
    else:
        _prepare_adamw(case, g, st)
    return st


def _prepare_attention(case, g, st):
    H, K, hd, t = case["heads"], case["kv"], case["hd"], TYPES[case["dtype"]]
    st["lk"], st["lq"] = _key_lengths(case), _query_lengths(case)
    # in any order
    order = torch.randperm(case["seqs"], generator=g, device=DEV).tolist()
    st["lk"], st["lq"] = [st["lk"][i] for i in order], [st["lq"][i] for i in order]
    st["sk"], st["nk"] = _places(st["lk"], case["room"])
    st["sq"], st["nq"] = _places(st["lq"], case["room"])
    st["scale"] = SCALE_OF_SCORES / math.sqrt(hd)
    if case["queries"]:
        st["q"] = _randn(g, st["nq"], H * hd, dtype=t)
        kv = _randn(g, st["nk"], 2 * K * hd, dtype=t)
        st["k"], st["v"] = kv[:, :K * hd], kv[:, K * hd:]
    else:
        # one projection's output holds all three
        qkv = _randn(g, st["nq"], (H + 2 * K) * hd, dtype=t)
        st["q"], st["k"], st["v"] = qkv[:, :H * hd], qkv[:, H * hd:(H + K) * hd], qkv[:, (H + K) * hd:]
    tensor = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    st["q_starts"], st["k_starts"] = tensor(st["sq"]), tensor(st["sk"])
    st["q_lens"], st["k_lens"] = tensor(st["lq"]), tensor(st["lk"])
    st["out"], st["lse"] = _zeros(st["nq"], H * hd, dtype=t), _zeros(H, st["nq"])
    if case["kind"] == "attention_backward":
        st["out"], st["lse"] = _plain_attention(st)
        st["dout"] = _randn(g, st["nq"], H * hd, dtype=t, scale=0.1)
        if case["queries"]:
            st["dq"] = _zeros(st["nq"], H * hd, dtype=t)
            dkv = _zeros(st["nk"], 2 * K * hd, dtype=t)
            st["dk"], st["dv"] = dkv[:, :K * hd], dkv[:, K * hd:]
        else:
            d = _zeros(st["nq"], (H + 2 * K) * hd, dtype=t)
            st["dq"], st["dk"], st["dv"] = d[:, :H * hd], d[:, H * hd:(H + K) * hd], d[:, (H + K) * hd:]
    if own:
        import paper_2608_11226_amd as R

        st["shape"] = R.AttentionShape(dtype=R.DTYPE_FP32 if case["dtype"] == "fp32" else R.DTYPE_BF16, n_heads=H, n_kv_heads=K, head_dim=hd,
                                       n_seqs=case["seqs"], n_q=st["nq"], n_k=st["nk"], causal=int(case["causal"]), scale=st["scale"])
        ask = R.rollout_attention_backward_workspace if case["kind"] == "attention_backward" else R.rollout_attention_workspace
        st["bytes"] = ask(st["shape"])
        st["ws"] = _zeros(max(1, st["bytes"]), dtype=torch.uint8)


def _prepare_adamw(case, g, st):
    """Every tensor a run of whole blocks in one buffer for the weights, one for the gradients, one for each state."""
    sizes = _adamw_sizes(case)
    blocks = [-(-n // BLOCK) for n in sizes]
    nb = sum(blocks)
    t = torch.tensor(blocks, device=DEV)
    st["tensor"] = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), t)  # a block's tensor
    st["first"] = (torch.arange(nb, device=DEV) - (torch.cumsum(t, 0) - t)[st["tensor"]]) * BLOCK  # its first element there
    left = torch.tensor(sizes, device=DEV)[st["tensor"]] - st["first"]
    there = torch.arange(BLOCK, device=DEV)[None] < left[:, None]
    st["decay"] = torch.tensor([0.0 if n == case["d"] else DECAY for n in sizes], device=DEV)
    # keys of the hash as two's complement
    st["keys"] = torch.tensor([k - (1 << 64) if k >> 63 else k for k in map(_tensor_key, range(len(sizes)))], device=DEV)
    p = _randn(g, nb, BLOCK, scale=0.02) * there
    # a state that some steps have left behind: gradients differ widely from element to element
    size = torch.exp(2.0 * _randn(g, nb, BLOCK)) * 1e-4
    grad = _randn(g, nb, BLOCK) * size * there
    m, v = 0.4 * _randn(g, nb, BLOCK) * size * there, (0.3 + torch.rand((nb, BLOCK), generator=g, device=DEV)) * size.square() * there
    st["p"], st["g"] = p.to(TYPES[case["param"]]), grad.to(TYPES[case["grad"]])
    del p, grad, size, there
    if case["state"] == "e4m3":
        st["m"], st["ms"] = _encode(m)
        st["v"], st["vs"] = _encode(torch.sqrt(v))
    else:
        st["m"], st["v"], st["ms"], st["vs"] = m, v, None, None
    st["copy"] = st["p"].to(torch.bfloat16) if case["copy"] else None
    st["grad_scale"] = torch.full((1,), 0.75, device=DEV)
    if own:
        import paper_2608_11226_amd as R

        flat = {k: st[k].view(-1) for k in ("p", "g", "m", "v", "copy") if st[k] is not None}
        tensors, at = [], 0
        for n, b in zip(sizes, blocks):
            view = lambda k: flat[k][at * BLOCK:at * BLOCK + n] if k in flat else None  # noqa: B023, E731
            scale = lambda k: None if st[k] is None else st[k][at:at + b]  # noqa: B023, E731
            tensors.append(R.adamw_tensor(view("p"), view("g"), view("m"), view("v"), 0.0 if n == case["d"] else DECAY,
                                          m_scales=scale("ms"), v_scales=scale("vs"), copy=view("copy")))
            at += b
        table, st["chunks"] = R.rollout_adamw_table(tensors)
        st["table"], st["tensors"] = table.to(DEV), len(tensors)


def _power(amax):
    """The smallest power of two that brings amax to at most 448 (2^-126 at least)."""
    f, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 9 + (f > 0.875).to(e.dtype), -126)
    return torch.ldexp(torch.ones_like(amax), torch.clamp(e, min=-126))


def _encode(x):
    """Nearest e4m3 of blocks."""
    s = _power(x.abs().amax(1))
    return (x / s[:, None]).to(E4M3), s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(st):
    kind = st["case"]["kind"]
    return _own(kind, st) if own else PLAIN[kind](st)


def _own(kind, st):
    import paper_2608_11226_amd as R

    case = st["case"]
    code = {"fp32": R.DTYPE_FP32, "bf16": R.DTYPE_BF16, "e4m3": R.DTYPE_E4M3}
    stream = torch.cuda.current_stream().cuda_stream
    if kind.startswith("attention"):
        inputs = (st["q"], st["q"].stride(0), st["k"], st["k"].stride(0), st["v"], st["v"].stride(0),
                  st["q_starts"], st["q_lens"], st["k_starts"], st["k_lens"])
        if kind == "attention":
            R.rollout_attention(st["shape"], *inputs, st["out"], st["out"].stride(0), st["lse"], st["ws"], st["bytes"], stream)
            return [st["out"], st["lse"]]
        R.rollout_attention_backward(st["shape"], *inputs, st["out"], st["out"].stride(0), st["lse"], st["dout"], st["dout"].stride(0),
                                     st["dq"], st["dq"].stride(0), st["dk"], st["dk"].stride(0), st["dv"], st["dv"].stride(0),
                                     st["ws"], st["bytes"], stream)
        return [st["dq"], st["dk"], st["dv"]]
    if kind == "norm":
        R.rollout_rms_norm(st["x"], code[case["x"]], st["delta"], code[case["delta"] or "bf16"], st["gain"], case["rows"], case["dim"], EPS,
                           st["h"], st["y"], code[case["y"]], st["scales"], st["rstd"], stream)
        return [st["h"], st["y"], st["scales"], st["rstd"]]
    if kind == "norm_backward":
        R.rollout_rms_norm_backward(st["dy"], code[case["dy"]], st["h"], code[case["x"]], st["gain"], st["rstd"], case["rows"], case["dim"],
                                    st["inner"], st["dx"], code[case["dx"]], st["dgain"], 0, st["ws"], st["bytes"], stream)
        return [st["dx"], st["dgain"]]
    R.rollout_adamw(st["table"], st["tensors"], st["chunks"], HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], HYPER["step"],
                    HYPER["seed"], grad_scale=st["grad_scale"], stream=stream)
    return _adamw_outputs(st)


def _adamw_outputs(st):
    return [st["p"], st["m"], st["v"], st["ms"], st["vs"], st["copy"]]


def _scores(st, iq, ik):
    """q k^T times the scale of a padded batch, [sequences, kv heads, group, queries, keys], -inf where a key is not
    attended, and the padded q, k, v."""
    case = st["case"]
    H, K, hd = case["heads"], case["kv"], case["hd"]
    (rq, tq), (rk, tk) = iq, ik
    S, Lq, Lk = rq.shape[0], rq.shape[1], rk.shape[1]
    q = st["q"][rq].float().view(S, Lq, K, H // K, hd).permute(0, 2, 3, 1, 4).reshape(S, K, -1, hd)
    k = st["k"][rk].float().view(S, Lk, K, hd).transpose(1, 2).contiguous()
    v = st["v"][rk].float().view(S, Lk, K, hd).transpose(1, 2).contiguous()
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(st["scale"]).view(S, K, H // K, Lq, Lk)
    hidden = ~tk[:, None, :]
    if case["causal"]:
        last = torch.arange(Lq, device=DEV)[None] + tk.sum(1)[:, None] - tq.sum(1)[:, None]
        hidden = hidden | (torch.arange(Lk, device=DEV)[None, None] > last[:, :, None])
    return s.masked_fill_(hidden[:, None, None], -INF), q, k, v


def _unpad(x, index, out):
    """Rows [sequences, heads, rows, hd] of a padded batch into the rows of a packed matrix."""
    rows, there = index
    S, _, L, _ = x.shape
    out[rows[there]] = x.transpose(1, 2).reshape(S, L, -1)[there].to(out.dtype)
    return out


def _plain_attention(st):
    case = st["case"]
    H = case["heads"]
    iq, ik = _rows_index(st["sq"], st["lq"]), _rows_index(st["sk"], st["lk"])
    s, _, _, v = _scores(st, iq, ik)
    S, K, G, Lq, Lk = s.shape
    m = s.amax(4, keepdim=True)
    none = m == -INF
    p = torch.exp(s.sub_(m.masked_fill(none, 0.0)))
    l = p.sum(4, keepdim=True)
    o = torch.matmul(p.view(S, K, G * Lq, Lk), v).view(S, K, G, Lq, -1) / l.masked_fill(none, 1.0)
    lse = (m + torch.log(l))[..., 0].reshape(S, H, Lq)
    out = _unpad(o.reshape(S, H, Lq, -1), iq, torch.zeros_like(st["out"]))
    whole = torch.zeros_like(st["lse"])
    whole[:, iq[0][iq[1]]] = lse.transpose(0, 1)[:, iq[1]]
    return [out, whole]


def _plain_attention_backward(st):
    case = st["case"]
    H, K, hd = case["heads"], case["kv"], case["hd"]
    iq, ik = _rows_index(st["sq"], st["lq"]), _rows_index(st["sk"], st["lk"])
    s, q, k, v = _scores(st, iq, ik)
    S, _, G, Lq, Lk = s.shape
    lse = st["lse"][:, iq[0]].view(K, G, S, Lq).permute(2, 0, 1, 3)[..., None]
    p = torch.exp(s.sub_(lse.masked_fill(lse == -INF, 0.0)))
    # rows of padding have no gradient
    p.mul_(iq[1][:, None, None, :, None])
    grouped = lambda x: x[iq[0]].float().view(S, Lq, K, G, hd).permute(0, 2, 3, 1, 4).reshape(S, K, G * Lq, hd)  # noqa: E731
    do, o = grouped(st["dout"]), grouped(st["out"])
    D = (do * o).sum(3, keepdim=True)
    p = p.view(S, K, G * Lq, Lk)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_(D).mul_(p).mul_(st["scale"])
    dq = torch.matmul(ds, k).view(S, H, Lq, hd)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    new = lambda n, w: torch.zeros((n, w), device=DEV, dtype=st["q"].dtype)  # noqa: E731
    return [_unpad(dq, iq, new(st["nq"], H * hd)), _unpad(dk, ik, new(st["nk"], K * hd)), _unpad(dv, ik, new(st["nk"], K * hd))]


def _plain_norm(st):
    case = st["case"]
    h = st["x"].float()
    if case["delta"]:
        h = (h + st["delta"].float()).to(st["x"].dtype)
    stored = h if case["delta"] else None
    h = h.float()
    rstd = torch.rsqrt(h.square().mean(1) + EPS)
    y = h * rstd[:, None] * st["gain"]
    if case["y"] != "e4m3":
        return [stored, y.to(TYPES[case["y"]]), None, rstd]
    scales = _power(y.abs().amax(1))
    return [stored, (y / scales[:, None]).to(E4M3), scales, rstd]


def _plain_norm_backward(st):
    h, dy, r = st["h"].float(), st["dy"].float(), st["rstd"][:, None]
    xhat = h * r
    t = dy * st["gain"]
    dx = r * (t - xhat * (t * xhat).mean(1, keepdim=True))
    if st["inner"] is not None:
        dx = dx + st["inner"].float()
    return [dx.to(st["dx"].dtype), (dy * xhat).sum(0)]


def _random16(st):
    """Three times 16 bits for every element: for the first moment, the second, the weight."""
    low = lambda x: x & 0xFFFFFFFF  # noqa: E731

    def finish(h):
        h = low((h ^ (h >> 16)) * 0x85EBCA6B)
        h = low((h ^ (h >> 13)) * 0xC2B2AE35)
        return h ^ (h >> 16)

    key = st["keys"][st["tensor"]][:, None]
    i = st["first"][:, None] + torch.arange(BLOCK, device=DEV)[None]
    h = finish(low(i * 0x9E3779B1 + low(key)))
    return h & 0xFFFF, h >> 16, (finish(low(h + low(key >> 32))) & 0xFFFF) if st["case"]["param"] == "bf16" else None


def _towards(x, random16):
    """|x| <= 448 to one of the two neighbouring e4m3 values, the upper one as likely as x is near it."""
    a = x.abs()
    small = a < 2.0 ** -6
    z = torch.where(small, a + 2.0 ** -6, a).view(torch.int32)
    z = ((z + random16.to(torch.int32) * 16 + 8) & -(1 << 20)).view(torch.float32)
    return torch.copysign(torch.where(small, z - 2.0 ** -6, z), x)


def _plain_adamw(st):
    case = st["case"]
    b1, b2 = HYPER["beta1"], HYPER["beta2"]
    g = st["g"].float() * st["grad_scale"]
    eight = case["state"] == "e4m3"
    m = st["m"].float() * st["ms"][:, None] if eight else st["m"]
    v = (st["v"].float() * st["vs"][:, None]).square() if eight else st["v"]
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g.square()
    p = st["p"].float()
    decay = (1 - HYPER["lr"] * st["decay"])[st["tensor"]][:, None]
    root = torch.sqrt(v)
    step = HYPER["lr"] / (1 - b1 ** HYPER["step"])
    p = p * decay - step * m / (root * (1 / math.sqrt(1 - b2 ** HYPER["step"])) + HYPER["eps"])
    if eight or case["param"] == "bf16":
        rm, rv, rp = _random16(st)
    if eight:
        ms, vs = _power(m.abs().amax(1)), _power(root.amax(1))
        st["m"].copy_(_towards(m / ms[:, None], rm))
        code = _towards(root / vs[:, None], rv)
        st["v"].copy_(torch.where((code == 0) & (root > 0), 2.0 ** -9, code))
        st["ms"].copy_(ms)
        st["vs"].copy_(vs)
    else:
        st["m"].copy_(m)
        st["v"].copy_(v)
    if case["param"] == "bf16":
        bits = (p.view(torch.int32) + rp.to(torch.int32)) & -(1 << 16)
        p = bits.view(torch.float32)
    st["p"].copy_(p)
    if case["copy"]:
        st["copy"].copy_(p)
    return _adamw_outputs(st)


PLAIN = {"attention": _plain_attention, "attention_backward": _plain_attention_backward, "norm": _plain_norm,
         "norm_backward": _plain_norm_backward, "adamw": _plain_adamw}


# ---------------------------------------------------------------------------
# work
# ---------------------------------------------------------------------------
def _pairs(case):
    """Pairs of a query and a key that it attends, over all sequences."""
    if not case["causal"]:
        return sum(a * b for a, b in zip(_query_lengths(case), _key_lengths(case)))
    return sum(a * b - a * (a - 1) // 2 for a, b in zip(_query_lengths(case), _key_lengths(case)))


def work(case):
    kind = case["kind"]
    if kind.startswith("attention"):
        es = SIZE[case["dtype"]]
        nq, nk = sum(_query_lengths(case)), sum(_key_lengths(case))
        row, kv_row = case["heads"] * case["hd"], case["kv"] * case["hd"]
        f = 2 * _pairs(case) * case["heads"] * case["hd"]
        if kind == "attention":
            return {"bytes": es * (2 * nq * row + 2 * nk * kv_row) + 4 * nq * case["heads"], "flops": 2 * f}
        # q, out, dout in and dq out; k, v in and dk, dv out
        return {"bytes": es * (4 * nq * row + 4 * nk * kv_row) + 4 * nq * case["heads"], "flops": 5 * f}
    if kind == "norm":
        n, d = case["rows"], case["dim"]
        each = SIZE[case["x"]] + (SIZE[case["delta"]] + SIZE[case["x"]] if case["delta"] else 0) + SIZE[case["y"]]
        return {"bytes": n * d * each + 4 * d + n * (8 if case["y"] == "e4m3" else 4), "flops": n * d * 6}
    if kind == "norm_backward":
        n, d = case["rows"], case["dim"]
        each = SIZE[case["x"]] + SIZE[case["dy"]] + SIZE[case["dx"]] * (2 if case["inner"] else 1)
        return {"bytes": n * d * each + 8 * d + 4 * n, "flops": n * d * 10}
    n = sum(_adamw_sizes(case))
    each = 2 * SIZE[case["param"]] + SIZE[case["grad"]] + 4 * SIZE[case["state"]] + (2 if case["copy"] else 0)
    return {"bytes": n * each + (16 * n // BLOCK if case["state"] == "e4m3" else 0), "flops": n * 15}


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def _nearest_e4m3(x):
    """Nearest e4m3 value, ties to the even one, of |x| <= 448."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _power_exact(amax):
    e = torch.floor(torch.log2(amax.clamp(min=1e-300)))
    f = amax / torch.exp2(e)
    return torch.exp2(torch.clamp(e - 8 + (f > 1.75).double(), min=-126.0))


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("attention"):
        return _exact_attention(st, case, kind == "attention_backward")
    if kind == "norm":
        h = st["x"].double()
        if case["delta"]:
            # as it is stored (a sum of two 32-bit numbers is rounded once)
            h = (h + st["delta"].double()).to(st["x"].dtype).double()
        rstd = 1.0 / torch.sqrt((h * h).sum(1) / case["dim"] + EPS)
        y = h * rstd[:, None] * st["gain"].double()
        stored = h if case["delta"] else None
        if case["y"] != "e4m3":
            return [stored, y, None, rstd]
        s = _power_exact(y.abs().amax(1))
        return [stored, _nearest_e4m3(y / s[:, None]), s, rstd]
    if kind == "norm_backward":
        h, dy, r = st["h"].double(), st["dy"].double(), st["rstd"].double()[:, None]
        t = dy * st["gain"].double()
        dx = r * t - r ** 3 * h * ((t * h).sum(1, keepdim=True) / case["dim"])
        if case["inner"]:
            dx += st["inner"].double()
        return [dx, (dy * h * r).sum(0)]
    return _exact_adamw(st, case)


def _exact_attention(st, case, backward):
    H, K, hd, scale = case["heads"], case["kv"], case["hd"], st["scale"]
    G = H // K
    wide = lambda n, w: torch.zeros((n, w), device=DEV, dtype=torch.float64)  # noqa: E731
    if backward:
        dq, dk, dv = wide(st["nq"], H * hd), wide(st["nk"], K * hd), wide(st["nk"], K * hd)
    else:
        out, lse = wide(st["nq"], H * hd), wide(H, st["nq"])
    for q0, nq, k0, nk in zip(st["sq"], st["lq"], st["sk"], st["lk"]):
        hide = torch.zeros((nq, nk), device=DEV, dtype=torch.bool)
        if case["causal"]:
            hide = torch.arange(nk, device=DEV)[None] > (torch.arange(nq, device=DEV) + nk - nq)[:, None]
        for h in range(H):
            a, b = slice(h * hd, h * hd + hd), slice(h // G * hd, h // G * hd + hd)
            q, k, v = st["q"][q0:q0 + nq, a].double(), st["k"][k0:k0 + nk, b].double(), st["v"][k0:k0 + nk, b].double()
            s = (q @ k.t()) * scale
            s[hide] = -INF
            if not backward:
                z = torch.logsumexp(s, 1)
                lse[h, q0:q0 + nq] = z
                out[q0:q0 + nq, a] = torch.nan_to_num(torch.exp(s - z[:, None])) @ v
                continue
            p = torch.nan_to_num(torch.exp(s - st["lse"][h, q0:q0 + nq].double()[:, None]))
            do, o = st["dout"][q0:q0 + nq, a].double(), st["out"][q0:q0 + nq, a].double()
            ds = p * (do @ v.t() - (do * o).sum(1, keepdim=True)) * scale
            dq[q0:q0 + nq, a] = ds @ k
            dk[k0:k0 + nk, b] += ds.t() @ q
            dv[k0:k0 + nk, b] += p.t() @ do
    return [dq, dk, dv] if backward else [out, lse]


def _exact_adamw(st, case):
    b1, b2, t = HYPER["beta1"], HYPER["beta2"], HYPER["step"]
    eight = case["state"] == "e4m3"
    g = st["g"].double() * 0.75
    m, v = st["m"].double(), st["v"].double()
    if eight:
        m *= st["ms"].double()[:, None]
        v *= st["vs"].double()[:, None]
        v *= v
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    p = st["p"].double()
    p -= HYPER["lr"] * (p * st["decay"].double()[st["tensor"]][:, None] + m / (1 - b1 ** t) / (torch.sqrt(v / (1 - b2 ** t)) + HYPER["eps"]))
    rounding = _random16(st) if eight or case["param"] == "bf16" else None
    ms = vs = None
    if eight:
        v = torch.sqrt(v)
        ms, vs = _power_exact(m.abs().amax(1)), _power_exact(v.amax(1))

        def stored(x, bits):
            a = x.abs()
            step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
            return torch.sign(x) * torch.floor(a / step + (16 * bits + 8).double() / 2 ** 20) * step

        m = stored(m / ms[:, None], rounding[0])
        some = v > 0
        v = torch.maximum(stored(v / vs[:, None], rounding[1]), some.double() * 2.0 ** -9)
    if case["param"] == "bf16":
        step = torch.exp2(torch.floor(torch.log2(p.abs().clamp(min=2.0 ** -126))) - 7)
        p = torch.sign(p) * torch.floor(p.abs() / step + rounding[2].double() / 2 ** 16) * step
    return [p, m, v, ms, vs, p if case["copy"] else None]
