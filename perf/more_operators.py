"""What the layers of a decoder are made of that a beam search steps: products with weights of 4 bits, and the gated delta rule.

A case is a dict of plain values.  Kinds:

  quantize  a matrix of weights to codes of 4 bits with a scale (and a zero) for each row and group of inputs, and the values
            that these stand for read back, as a loader does that looks at what rounding lost;
  linear    rows times such a matrix, plus a bias and rows to be added;
  gated     act(rows times one matrix) * (rows times another): the first half of a gated feed-forward block;
  delta     the gated delta rule over new tokens of rows, each from the state that its parent left: one token (a step) or many
            (prompts).

Codes lie as [ceil(N / 16), ceil(K / 128), 4, 16, 16] bytes: 16 outputs and 128 inputs at a time, of them the c-th eight of
every 32, an output, four words of 32 bits (one for each 32 inputs).  Byte i of a word holds input i of its eight in the lower and input
i + 4 in the upper four bits.
Scales [ceil(N / 16), ceil(K / 128), 16, 128 / group] of 16 bits, zeros the same in bytes: those of an output's groups of 128 inputs
side by side; a value is (code - zero) * scale, the zero 8 where there are none.

With `own` false the operators are computed from their formulas with elementary torch operations, otherwise by the package.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
PLACES = (0, 4, 1, 5, 2, 6, 3, 7)                    # the input of each four bits of a word, the lowest bits first


def _quantize(name, N, K, group, dtype, scale="f16", zeros=False):
    return {"name": name, "kind": "quantize", "N": N, "K": K, "group": group, "dtype": dtype, "scale": scale, "zeros": zeros}


def _linear(name, M, N, K, group, dtype, out=None, scale="f16", zeros=False, bias=False, add=False):
    """out: the result's type, the rows' own unless given."""
    return {"name": name, "kind": "linear", "M": M, "N": N, "K": K, "group": group, "dtype": dtype, "out": out or dtype, "scale": scale,
            "zeros": zeros, "bias": bias, "add": add}


def _gated(name, M, N, K, group, dtype, act="silu", scale="f16", zeros=False):
    return {"name": name, "kind": "gated", "M": M, "N": N, "K": K, "group": group, "dtype": dtype, "act": act, "scale": scale, "zeros": zeros}


def _delta(name, S, B, T, heads, k_heads, Dk, Dv, dtype, ragged=False, fresh=False):
    """T: new tokens of the longest row; fresh: rows begin with no state."""
    return {"name": name, "kind": "delta", "S": S, "B": B, "T": T, "heads": heads, "k_heads": k_heads, "Dk": Dk, "Dv": Dv, "dtype": dtype,
            "ragged": ragged, "fresh": fresh}


def listed():
    return [
        # sizes that are multiples of nothing, groups of 32 with zeros
        _quantize("quantize, odd", 1023, 1500, 32, "f32", scale="bf16", zeros=True),
        # a large projection, as it is loaded
        _quantize("quantize, large", 16384, 4096, 128, "bf16"),
        # the smallest projection that anybody steps, one row: nothing but latency
        _linear("linear, one row", 1, 1024, 1024, 128, "bf16"),
        # a projection of a step of one sentence's beams, on top of what went by
        _linear("linear, beams", 12, 4096, 4096, 128, "bf16", add=True),
        # the translation model's output layer, logits in fp32
        _linear("linear, output layer", 12, 40000, 1000, 32, "f32", scale="bf16", zeros=True, bias=True),
        # prompts of a batch
        _linear("linear, prompts", 2048, 8192, 8192, 128, "f16"),
        # a step of a batch with a few beams each
        _gated("gated, beams", 40, 16384, 4096, 128, "bf16"),
        # multiples of nothing, rows in fp32, the other activation
        _gated("gated, odd", 150, 5001, 1900, 64, "f32", act="gelu", scale="bf16", zeros=True),
        # a step of one sentence's beams
        _delta("delta, one sentence", 1, 12, 1, 8, 8, 64, 64, "f32"),
        # a step of a batch of beams
        _delta("delta, batch", 32, 10, 1, 16, 8, 128, 128, "bf16"),
        # prompts of a batch, odd heads
        _delta("delta, prompts", 12, 1, 700, 12, 6, 96, 160, "f16", ragged=True),
        # one long prompt
        _delta("delta, long prompt", 1, 1, 8192, 16, 16, 128, 128, "bf16", fresh=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_once(rng):
    kind = rng.choice(["quantize"] + ["linear"] * 4 + ["gated"] * 2 + ["delta"] * 4)
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind == "delta":
        k_heads = rng.choice([1, 2, 4, 8, 16])
        T = rng.choice([1, 1, rng.randint(2, 16), _log_int(rng, 16, 8192), _log_int(rng, 16, 8192)])
        Dk, Dv = (rng.choice([32, 48, 64, 64, 80, 96, 128, 128, 128, 192, 256]) for _ in range(2))
        return _delta(None, _log_int(rng, 1, 32), rng.choice([1, 1, 4, 10, 12]) if T <= 16 else 1, T, k_heads * rng.choice([1, 1, 2, 3]), k_heads,
                      Dk, Dv if rng.random() < 0.4 else Dk, dtype, rng.random() < 0.5, rng.random() < 0.4)
    N, K = (rng.choice([x, x, x // 64 * 64 + 64]) for x in (_log_int(rng, 64, 40000), _log_int(rng, 64, 16384)))
    group, scale, zeros = rng.choice([32, 64, 128]), rng.choice(["f16", "bf16"]), rng.random() < 0.4
    if kind == "quantize":
        return _quantize(None, N, K, group, dtype, scale, zeros)
    M = rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 1, 64), _log_int(rng, 16, 2048)])
    if kind == "gated":
        return _gated(None, M, N, K, group, dtype, rng.choice(["silu", "silu", "gelu", "gelu_tanh"]), scale, zeros)
    return _linear(None, M, N, K, group, dtype, rng.choice([dtype, dtype, "f32"]), scale, zeros, rng.random() < 0.3, rng.random() < 0.4)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw_once(rng)
        # what a call has in memory and its plain form in fp32
        state = c["S"] * c["B"] * c["heads"] * c["Dk"] * c["Dv"] if c["kind"] == "delta" else c["N"] * c["K"]
        rows = c["S"] * c["B"] * c["T"] * c["heads"] * max(c["Dk"], c["Dv"]) if c["kind"] == "delta" else 0
        if _cost(c) <= most and state <= 1.5e8 and rows <= 6e7:
            del c["name"]
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 3e14)


# ---- inputs -----------------------------------------------------------------------------------

def _randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def _weights(c, g):
    """Codes as rounding normal values leaves them, scales of a trained layer's size.  What stands behind the last output or
    input is never zeros: nobody clears it."""
    N, K = c["N"], c["K"]
    tiles, parts, each = -(-N // 16), -(-K // 128), 128 // c["group"]
    low, high = ((_randn(g, tiles, parts, 4, 16, 16) * 2.6).round_().clamp_(-7, 7).to(torch.int8) + 8 for _ in range(2))
    codes = (low + high * 16).view(torch.uint8)
    scales = (torch.exp(_randn(g, tiles, parts, 16, each) * 0.4) * (0.4 / math.sqrt(K))).to(DTYPES[c["scale"]])
    zeros = torch.randint(4, 12, (tiles, parts, 16, each), device="cuda", generator=g).to(torch.uint8) if c["zeros"] else None
    return {"codes": codes, "scales": scales, "zeros": zeros}


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed * 16 + 1)
    rng = np.random.default_rng(seed)
    st = {"case": c}
    if c["kind"] == "delta":
        S, B, T, H = c["S"], c["B"], c["T"], c["heads"]
        R, dtype = S * B, DTYPES[c["dtype"]]
        # queries, keys and values as one projection leaves them, the first two of unit length
        q, k = (_randn(g, R, T, c["k_heads"], c["Dk"]) for _ in range(2))
        q, k = (x / x.square().sum(-1, keepdim=True).sqrt() for x in (q, k))
        v = _randn(g, R, T, H, c["Dv"])
        row = torch.cat([x.flatten(2) for x in (q, k, v)], 2).to(dtype)
        nk, nv = c["k_heads"] * c["Dk"], H * c["Dv"]
        st["q"], st["k"], st["v"] = (x.unflatten(2, (n, -1)) for x, n in zip(row.split([nk, nk, nv], 2), (c["k_heads"], c["k_heads"], H)))
        rate = torch.exp(torch.rand(H, device="cuda", generator=g) * 5.0 - 3.5)           # heads forget at different rates
        st["decay"] = (-rate * torch.log1p(torch.exp(_randn(g, R, T, H) - 2.0))).contiguous()
        st["beta"] = torch.sigmoid(_randn(g, R, T, H) * 1.5)
        new = np.full(R, T)
        if c["ragged"]:
            new = np.maximum(1, np.round(T * rng.random(R) ** 1.5)).astype(np.int64)
            new[rng.integers(R)] = T
        st["new"] = torch.from_numpy(new.astype(np.int32)).cuda()
        st["state"] = st["parents"] = None
        if not c["fresh"]:
            st["state"] = _randn(g, R, H, c["Dk"], c["Dv"]) * 0.3
            st["parents"] = torch.from_numpy(np.sort(rng.integers(0, B, (S, B)), axis=1).reshape(-1).astype(np.int32)).cuda()
        st["state_out"] = torch.empty(R, H, c["Dk"], c["Dv"], dtype=torch.float32, device="cuda")
        st["out"] = torch.zeros(R, T, H, c["Dv"], dtype=dtype, device="cuda")             # rows behind a row's last token stay
        return st
    if c["kind"] == "quantize":
        N, K = c["N"], c["K"]
        tiles, parts, each = -(-N // 16), -(-K // 128), 128 // c["group"]
        st["w"] = (_randn(g, N, K) * torch.exp(_randn(g, N, 1) * 0.3) * (1.0 / math.sqrt(K))).to(DTYPES[c["dtype"]])
        st["codes"] = torch.zeros(tiles, parts, 4, 16, 16, dtype=torch.uint8, device="cuda")
        st["scales"] = torch.zeros(tiles, parts, 16, each, dtype=DTYPES[c["scale"]], device="cuda")
        st["zeros"] = torch.zeros(tiles, parts, 16, each, dtype=torch.uint8, device="cuda") if c["zeros"] else None
        st["values"] = torch.empty_like(st["w"])
        return st
    M, N, K = c["M"], c["N"], c["K"]
    # activations: a few inputs are far larger than the others
    size = torch.where(torch.rand(K, device="cuda", generator=g) < 0.01, 12.0, 1.0)
    st["x"] = (_randn(g, M, K) * size).to(DTYPES[c["dtype"]])
    if c["kind"] == "gated":
        st["gate"], st["up"] = _weights(c, g), _weights(c, g)
        st["out"] = torch.empty(M, N, dtype=DTYPES[c["dtype"]], device="cuda")
        return st
    st["w"] = _weights(c, g)
    st["bias"] = _randn(g, N) * 0.5 if c["bias"] else None
    st["add"] = _randn(g, M, N).to(DTYPES[c["out"]]) if c["add"] else None
    st["out"] = torch.empty(M, N, dtype=DTYPES[c["out"]], device="cuda")
    return st


# ---- the plain forms --------------------------------------------------------------------------

def _unpacked(codes, N, K):
    """[N, K] codes as numbers."""
    both = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)           # [tiles, parts, 4, 16, 32]: places in order
    both = both.unflatten(-1, (4, 8))[..., torch.tensor([PLACES.index(i) for i in range(8)], device="cuda")]
    both = both.permute(0, 3, 1, 4, 2, 5).flatten(2)                       # [tiles, output, parts * word * part of 32 * input]
    return both.flatten(0, 1)[:N, :K]


def _packed(codes, tiles, parts):
    """The other way round: codes [N, K] as they lie, 0 behind the last."""
    both = torch.zeros(16 * tiles, 128 * parts, dtype=torch.uint8, device="cuda")
    both[:codes.shape[0], :codes.shape[1]] = codes
    both = both.view(tiles, 16, parts, 4, 4, 8).permute(0, 2, 4, 1, 3, 5)[..., torch.tensor(PLACES, device="cuda")]
    return (both[..., 0::2] | both[..., 1::2] << 4).flatten(-2).contiguous()


def _of_groups(x, c):
    """[N, groups] numbers of a tensor of scales or zeros."""
    return x.permute(0, 2, 1, 3).flatten(2).flatten(0, 1)[:c["N"], :-(-c["K"] // c["group"])].float()


def _to_groups(x, to):
    """The other way round, as they lie, 0 behind the last."""
    all_of = torch.zeros(16 * to.shape[0], to.shape[1] * to.shape[3], dtype=x.dtype, device="cuda")
    all_of[:x.shape[0], :x.shape[1]] = x
    to.copy_(all_of.view(to.shape[0], 16, to.shape[1], to.shape[3]).permute(0, 2, 1, 3))


def _values(w, c):
    N, K, group = c["N"], c["K"], c["group"]
    scale = _of_groups(w["scales"], c)
    zero = _of_groups(w["zeros"], c) if w["zeros"] is not None else torch.full_like(scale, 8.0)
    part = torch.arange(K, device="cuda") // group
    return (_unpacked(w["codes"], N, K).float() - zero[:, part]) * scale[:, part]


def _act(x, name):
    if name == "silu":
        return x / (1 + torch.exp(-x))
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))


def _quantize_plain(st, c):
    N, K, group = c["N"], c["K"], c["group"]
    groups, tiles, parts = -(-K // group), -(-N // 16), -(-K // 128)
    w = torch.zeros(N, groups * group, device="cuda")
    w[:, :K] = st["w"]
    w = w.view(N, groups, group)
    if c["zeros"]:
        lo, hi = w.amin(2).clamp(max=0).double(), w.amax(2).clamp(min=0).double()
        scale = (hi - lo) / 15
    else:
        scale = w.abs().amax(2).double() / 7
    # (what is next to a border: 64 bits; the scale rounded to 32 bits and then to 16)
    scale = scale.to(DTYPES[c["scale"]])
    s = torch.where(scale > 0, scale.double(), torch.full_like(scale, math.inf, dtype=torch.float64))
    zero = (-lo / s).round().clamp(0, 15) if c["zeros"] else torch.full_like(s, 8.0)
    code = ((w / s[..., None]).round() + zero[..., None]).clamp(0, 15).to(torch.uint8).flatten(1)[:, :K]
    st["codes"].copy_(_packed(code, tiles, parts))
    _to_groups(scale, st["scales"])
    if c["zeros"]:
        _to_groups(zero, st["zeros"])
    st["values"].copy_(_values(st, c))
    return _quantized(st, c)


def _quantized(st, c):
    out = {"values": st["values"], "scales": st["scales"]}
    if c["zeros"]:
        out["zeros"] = st["zeros"]
    return out


def _linear_plain(st, c):
    y = torch.matmul(st["x"].float(), _values(st["w"], c).t())
    if c["bias"]:
        y = y + st["bias"]
    if c["add"]:
        y = y + st["add"].float()
    st["out"].copy_(y)
    return st["out"]


def _gated_plain(st, c):
    x = st["x"].float()
    st["out"].copy_(_act(torch.matmul(x, _values(st["gate"], c).t()), c["act"]) * torch.matmul(x, _values(st["up"], c).t()))
    return st["out"]


def _begin(st, c):
    """The states that rows begin with."""
    S, B = c["S"], c["B"]
    if c["fresh"]:
        return torch.zeros_like(st["state_out"])
    return st["state"][torch.arange(S * B, device="cuda") // B * B + st["parents"].long()]


def _delta_plain(st, c):
    """64 tokens at a time: what their keys ask of the state and of each other is a triangular system."""
    T, H, C = c["T"], c["heads"], min(64, c["T"])
    live = torch.arange(T, device="cuda")[None, :, None] < st["new"][:, None, None]
    share = H // c["k_heads"]
    q, k = (st[n].float().transpose(1, 2).repeat_interleave(share, 1) for n in ("q", "k"))          # [R, H, T, Dk]
    v = st["v"].float().transpose(1, 2)
    g = torch.where(live, st["decay"], 0.0).transpose(1, 2)
    b = torch.where(live, st["beta"], 0.0).transpose(1, 2)
    S = _begin(st, c)
    seen = torch.ones(C, C, dtype=torch.bool, device="cuda").tril()
    out = []
    for at in range(0, T, C):
        n = min(C, T - at)
        qc, kc, vc, bc = (x[:, :, at:at + n] for x in (q, k, v, b))
        sums = g[:, :, at:at + n].double().cumsum(2)
        apart = torch.where(seen[:n, :n], (sums[..., :, None] - sums[..., None, :]).exp().float(), 0.0)
        e = sums.exp().float()[..., None]
        kt = kc.transpose(2, 3).contiguous()
        system = bc[..., None] * (apart * torch.matmul(kc, kt)).tril(-1)
        right = bc[..., None] * (vc - e * torch.matmul(kc, S))
        u, power = right, -system                                          # (1 + system)^-1 = ... (1 + system^4) (1 + system^2) (1 - system)
        for _ in range((n - 1).bit_length()):
            u, power = u + torch.matmul(power, u), torch.matmul(power, power)
        out.append(e * torch.matmul(qc, S) + torch.matmul(apart * torch.matmul(qc, kt), u))
        last = (sums[..., -1:] - sums).exp().float()[..., None]
        S = e[..., -1:, :] * S + torch.matmul((last * kc).transpose(2, 3).contiguous(), u)
    o = torch.cat(out, 2).transpose(1, 2) / math.sqrt(c["Dk"])
    st["out"].copy_(torch.where(live[..., None], o, st["out"].float()))
    st["state_out"].copy_(S)
    return {"out": st["out"], "state": st["state_out"]}


# ---- the package's calls ----------------------------------------------------------------------

def _handles(st, c):
    """What a program keeps between calls: parameters, weights' handles, workspaces."""
    from paper_1806_00588_amd import binding

    def room(n):
        return torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")

    h = {"lib": binding}
    if c["kind"] == "delta":
        h["dp"] = binding.delta_params(c["S"], c["B"], c["T"], c["heads"], c["k_heads"], c["Dk"], c["Dv"], scale=1.0 / math.sqrt(c["Dk"]))
        h["ws"] = room(binding.delta_workspace_bytes(h["dp"]))
        return h
    h["pp"] = binding.packed_params(c["N"], c["K"], c["group"])
    for name in ("gate", "up") if c["kind"] == "gated" else ("w",):
        w = st if c["kind"] == "quantize" else st[name]
        h[name] = binding.PackedWeights(h["pp"], codes=w["codes"], scales=w["scales"], zeros=w["zeros"])
    if c["kind"] != "quantize":
        h["ws"] = room(binding.packed_workspace_bytes(h["pp"], c["M"]))
    return h


def _run_own(st, c):
    h = st.get("handles")
    if h is None:
        h = st["handles"] = _handles(st, c)
    lib = h["lib"]
    if c["kind"] == "quantize":
        lib.packed_quantize(h["pp"], st["w"], h["w"])
        lib.packed_values(h["pp"], h["w"], st["values"])
        return _quantized(st, c)
    if c["kind"] == "linear":
        lib.packed_linear(h["pp"], h["w"], st["x"], h["ws"], st["out"], bias=st["bias"], add=st["add"])
        return st["out"]
    if c["kind"] == "gated":
        lib.packed_gated(h["pp"], h["gate"], h["up"], st["x"], h["ws"], st["out"], act=c["act"])
        return st["out"]
    lib.delta_rule(h["dp"], st["q"], st["k"], st["v"], st["decay"], st["beta"], st["state"], st["state_out"], h["ws"], st["out"],
                   parents=st["parents"], n_new=st["new"])
    return {"out": st["out"], "state": st["state_out"]}


def run(state):
    c = state["case"]
    if own:
        return _run_own(state, c)
    return {"quantize": _quantize_plain, "linear": _linear_plain, "gated": _gated_plain, "delta": _delta_plain}[c["kind"]](state, c)


# ---- the same from the definitions, in 64 bits -------------------------------------------------

def _exact_matrix(w, c):
    """Values [N, K], word by word of the codes as they lie."""
    N, K, group = c["N"], c["K"], c["group"]
    words = w["codes"].view(torch.int32)                                   # [tiles, parts, 4, 16, 4]
    m = torch.zeros(16 * words.shape[0], 128 * words.shape[1], dtype=torch.float64, device="cuda")
    to = m.view(words.shape[0], 16, words.shape[1], 4, 4, 8)               # [tiles, output, parts, word, c, input]
    for place, i in enumerate(PLACES):
        to[..., i] = (words >> (4 * place) & 15).double().permute(0, 3, 1, 4, 2)
    m = m[:N, :K]
    each = 128 // group
    for at in range(-(-K // group)):
        part = m[:, at * group:(at + 1) * group]
        part -= w["zeros"][:, at // each, :, at % each].reshape(-1, 1)[:N].double() if w["zeros"] is not None else 8.0
        part *= w["scales"][:, at // each, :, at % each].reshape(-1, 1)[:N].double()
    return m


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    if c["kind"] == "quantize":
        N, K, group = c["N"], c["K"], c["group"]
        tiles, parts, _, each = st["scales"].shape
        scales, zeros = (torch.zeros(16 * tiles, parts * each, dtype=torch.float64, device="cuda") for _ in range(2))
        values = torch.zeros(N, K, dtype=torch.float64, device="cuda")
        for at in range(-(-K // group)):
            part = st["w"][:, at * group:(at + 1) * group].double()
            if c["zeros"]:
                least, most = torch.clamp(part.amin(1), max=0), torch.clamp(part.amax(1), min=0)
                step = ((most - least) / 15).to(DTYPES[c["scale"]]).double()
                zero = torch.clamp(torch.round(torch.nan_to_num(-least / step)), 0, 15)
                zeros[:N, at] = zero
                lowest, highest = -zero, 15 - zero
            else:
                step = (part.abs().amax(1) / 7).to(DTYPES[c["scale"]]).double()
                lowest, highest = torch.full_like(step, -8), torch.full_like(step, 7)
            whole = torch.round(torch.nan_to_num(part / step[:, None]))
            values[:, at * group:(at + 1) * group] = torch.minimum(torch.maximum(whole, lowest[:, None]), highest[:, None]) * step[:, None]
            scales[:N, at] = step
        scales, zeros = (x.view(tiles, 16, parts, each).transpose(1, 2) for x in (scales, zeros))
        return {"values": values, "scales": scales, "zeros": zeros} if c["zeros"] else {"values": values, "scales": scales}
    if c["kind"] == "linear":
        y = torch.matmul(st["x"].double(), _exact_matrix(st["w"], c).t())
        if st["bias"] is not None:
            y += st["bias"].double()
        if st["add"] is not None:
            y += st["add"].double()
        return y
    if c["kind"] == "gated":
        x = st["x"].double()
        a, b = torch.matmul(x, _exact_matrix(st["gate"], c).t()), torch.matmul(x, _exact_matrix(st["up"], c).t())
        if c["act"] == "silu":
            a = a * torch.sigmoid(a)
        elif c["act"] == "gelu":
            a = a * 0.5 * torch.erfc(-a / math.sqrt(2.0))
        else:
            a = a * torch.sigmoid(2.0 * math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3))
        return a * b
    # token by token
    R, T, H = c["S"] * c["B"], c["T"], c["heads"]
    head = torch.arange(H, device="cuda") // (H // c["k_heads"])
    if c["fresh"]:
        S = torch.zeros(R, H, c["Dk"], c["Dv"], dtype=torch.float64, device="cuda")
    else:
        S = torch.stack([st["state"][r // c["B"] * c["B"] + p] for r, p in enumerate(st["parents"].tolist())]).double()
    out = torch.zeros(R, T, H, c["Dv"], dtype=torch.float64, device="cuda")
    order = st["new"].argsort(descending=True, stable=True)
    new, S = st["new"][order].tolist(), S[order]
    for t in range(T):
        n = sum(x > t for x in new)                                        # the longest rows come first
        if n == 0:
            break
        rows = order[:n]
        k, q, v = st["k"][rows, t].double()[:, head], st["q"][rows, t].double()[:, head], st["v"][rows, t].double()
        state = S[:n] * st["decay"][rows, t].double().exp()[..., None, None]
        u = (v - (k[..., None] * state).sum(2)) * st["beta"][rows, t].double()[..., None]
        state += k[..., None] * u[:, :, None]
        S[:n] = state
        out[rows, t] = (q[..., None] * state).sum(2) / math.sqrt(c["Dk"])
    state = torch.empty_like(S)
    state[order] = S
    return {"out": out, "state": state}


# ---- what a pass cannot do without -------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "delta":
        R, H, Dk, Dv = c["S"] * c["B"], c["heads"], c["Dk"], c["Dv"]
        # ragged rows have 0.4 of the longest on average, the longest among them
        tokens = c["T"] * ((1 + 0.4 * (R - 1)) if c["ragged"] else R)
        state = 4.0 * R * H * Dk * Dv * (1 if c["fresh"] else 2)
        e = SIZE[c["dtype"]]
        return {"bytes": state + tokens * (e * (2 * c["k_heads"] * Dk + 2 * H * Dv) + 8 * H), "flops": 6.0 * tokens * H * Dk * Dv}
    N, K = c["N"], c["K"]
    weights = N * K / 2 + (3 if c["zeros"] else 2) * N * -(-K // c["group"])
    if c["kind"] == "quantize":
        return {"bytes": float(2 * weights + 2 * N * K * SIZE[c["dtype"]]), "flops": 2.0 * N * K}
    M, e = c["M"], SIZE[c["dtype"]]
    if c["kind"] == "gated":
        return {"bytes": float(2 * weights + M * K * e + M * N * e), "flops": 4.0 * M * N * K}
    o = SIZE[c["out"]]
    return {"bytes": float(weights + M * K * e + M * N * o * (2 if c["add"] else 1) + (4 * N if c["bias"] else 0)), "flops": 2.0 * M * N * K}
