"""Weights of 4 bits against references in 64 bits: quantising (equal, bit for bit), reading back, rows times them, the first half of a gated block.

Tolerance of a sum of K products: every product is exact.  A group's sum, the sum of its inputs, and the sum over groups round group + groups + 12
times at most (the twelve: zero, scale, eight waves, bias, what is added), each by 2^-23 at most of what has been added up, and that is never more
than sum |x| (code + zero) scale + |bias| + |add|.  The result's own rounding comes on top."""
import numpy as np
import pytest

from oracle import layers

pytestmark = pytest.mark.gpu

TYPES = ("f32", "bf16", "f16")


def torch_type(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def on_gpu(x, dtype="f32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch_type(dtype)).cuda()


def in_64(x):
    return x.double().cpu().numpy()


def round16(name):
    import torch
    return lambda x: float(torch.tensor(float(x), dtype=torch.float32).to(torch_type(name)).double())


def half_step(y, dtype):
    """What rounding to dtype costs at most."""
    eps, least = {"f32": (2.0 ** -24, 2.0 ** -150), "bf16": (2.0 ** -8, 2.0 ** -134), "f16": (2.0 ** -11, 2.0 ** -25)}[dtype]
    return np.abs(y) * eps + least


class Weights:
    """A matrix of 4-bit weights, on the GPU and as values; what lies behind the last output and input is senseless."""

    def __init__(self, rng, N, K, group, scale="f16", zeros=False):
        from paper_1806_00588_amd import binding
        groups, tiles, parts = -(-K // group), -(-N // 16), -(-K // 128)
        self.N, self.K, self.group = N, K, group
        self.codes = rng.integers(0, 16, (N, K))
        r = round16(scale)
        self.scales = np.vectorize(r)(np.exp(rng.normal(size=(N, groups)) * 0.5) / np.sqrt(K))
        self.zeros = rng.integers(0, 16, (N, groups)) if zeros else np.full((N, groups), 8)
        all_codes = rng.integers(0, 16, (16 * tiles, 128 * parts))
        all_codes[:N, :K] = self.codes
        shape = (tiles, parts, 16, 128 // group)
        self.pp = binding.packed_params(N, K, group)
        self.on_gpu = binding.PackedWeights(self.pp, codes=on_gpu_bytes(layers.pack(all_codes)), scales=on_gpu(layers.of_groups(self.scales, shape, np.nan), scale),
                                            zeros=on_gpu_bytes(layers.of_groups(self.zeros, shape, 255)) if zeros else None)
        g = np.arange(K) // group
        self.values = layers.values(self.codes, self.scales, self.zeros, group)
        self.sizes = (self.codes + self.zeros[:, g]) * self.scales[:, g]

    def product(self, x):
        """(x W^T, the most that a sum can be off before it is rounded)."""
        with np.errstate(invalid="ignore", over="ignore"):
            return x @ self.values.T, (self.group + -(-self.K // self.group) + 12) * 2.0 ** -23 * (np.abs(x) @ self.sizes.T)


def on_gpu_bytes(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x.astype(np.uint8))).cuda()


def workspace(n):
    import torch
    return torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")


# ---- quantising ---------------------------------------------------------------------------------

def check_quantize(w, group, dtype, scale, zeros, pitch=0):
    """w: values that dtype has."""
    import torch
    from paper_1806_00588_amd import binding
    N, K = w.shape
    pp = binding.packed_params(N, K, group)
    held = torch.full((N, K + pitch), 3.0, dtype=torch_type(dtype), device="cuda")
    held[:, :K] = on_gpu(w, dtype)
    to = binding.PackedWeights(pp, scale_dtype=torch_type(scale), zeros=True if zeros else None)
    to.codes.fill_(0x5a)
    to.scales.fill_(7.0)
    binding.packed_quantize(pp, held[:, :K], to)
    codes, scales, zs = layers.quantize(in_64(held[:, :K]).astype(np.float32), group, round16(scale), zeros)
    assert np.array_equal(to.codes.cpu().numpy(), layers.pack(codes))
    assert np.array_equal(in_64(to.scales), layers.of_groups(scales, tuple(to.scales.shape)), equal_nan=True)
    if zeros:
        assert np.array_equal(to.zeros.cpu().numpy(), layers.of_groups(zs, tuple(to.zeros.shape)))
    for out_type in TYPES:
        out = torch.full((N, K + pitch), -5.0, dtype=torch_type(out_type), device="cuda")
        binding.packed_values(pp, to, out[:, :K])
        want = torch.from_numpy(layers.values(codes, scales, zs if zeros else np.full_like(zs, 8), group).astype(np.float32)).to(torch_type(out_type))
        assert torch.equal(out[:, :K].cpu().nan_to_num(9.0), want.nan_to_num(9.0)) and bool((out[:, K:] == -5).all())


@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (17, 129), (5, 31), (33, 300), (40, 1000)])
@pytest.mark.parametrize("dtype,scale,group,zeros", [("f32", "f16", 32, False), ("f32", "bf16", 64, True), ("bf16", "f16", 128, False), ("bf16", "bf16", 32, True),
                                                     ("f16", "f16", 64, True), ("f16", "bf16", 128, False), ("f32", "bf16", 128, True)])
def test_quantize(N, K, dtype, scale, group, zeros):
    rng = np.random.default_rng(N + K)
    check_quantize(rng.normal(size=(N, K)) * np.exp(rng.normal(size=(N, 1))), group, dtype, scale, zeros, pitch=K % 5)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("scale", ["f16", "bf16"])
def test_quantize_values_at_borders(scale, zeros):
    """Quotients that are halves exactly, and next to them; groups of zeros, of one sign, with a NaN or an infinity, far too large and small for fp16."""
    rng = np.random.default_rng(3)
    w = np.zeros((20, 128), dtype=np.float32)
    step = np.float32(0.75 if zeros else 1.25)
    w[0] = (np.arange(128) % 30 - 14) / 2 * step
    w[0, :2] = (7 * step, -8 * step) if zeros else (7 * step, -7 * step)
    w[1] = np.nextafter(w[0], np.float32(np.inf), dtype=np.float32)
    w[2] = np.nextafter(w[0], np.float32(-np.inf), dtype=np.float32)
    w[1:3, :2] = w[0, :2]
    w[4] = np.abs(rng.normal(size=128))
    w[5] = -w[4]
    w[6:9] = rng.normal(size=(3, 128))
    w[6, 5], w[7, 70], w[8, 127] = np.nan, np.inf, -np.inf
    w[9] = rng.normal(size=128) * 1e30
    w[10] = rng.normal(size=128) * 1e-30
    w[11] = rng.normal(size=128) * 1e-39
    w[12] = rng.normal(size=128) * 3e-7
    w[13, 3] = -2.0
    w[14] = 1e-45
    w[15] = rng.normal(size=128) * 1e38 / 4
    for group in (32, 64, 128):
        check_quantize(w, group, "f32", scale, zeros)


# ---- rows times weights -------------------------------------------------------------------------

def rows_of(rng, M, K, dtype):
    import torch
    x = rng.normal(size=(M, K)) * np.where(rng.random(K) < 0.02, 12.0, 1.0)
    return torch.from_numpy(x).to(torch_type(dtype)).double().numpy()


def check_linear(rng, M, w, dtype, out_type, bias=False, add=None, pitch=0):
    """add: "own" or "in place"."""
    import torch
    from paper_1806_00588_amd import binding
    N, K = w.N, w.K
    x = rows_of(rng, M, K, dtype)
    held = torch.full((M, K + pitch), float("nan"), dtype=torch_type(dtype), device="cuda")
    held[:, :K] = on_gpu(x, dtype)
    y, off = w.product(x)
    b = rng.normal(size=N).astype(np.float32) if bias else None
    out = torch.full((M, N + pitch), 77.0, dtype=torch_type(out_type), device="cuda")
    more = None
    if add:
        more = on_gpu(rng.normal(size=(M, N)), out_type)
        y, off = y + in_64(more), off + (w.group + 12) * 2.0 ** -23 * np.abs(in_64(more))
        if add == "in place":
            out[:, :N] = more
            more = out[:, :N]
    if bias:
        y, off = y + b, off + (w.group + 12) * 2.0 ** -23 * np.abs(b)
    ws = workspace(binding.packed_workspace_bytes(w.pp, M))
    binding.packed_linear(w.pp, w.on_gpu, held[:, :K], ws, out[:, :N], bias=None if b is None else on_gpu(b), add=more)
    got = in_64(out[:, :N])
    assert np.all(np.abs(got - y) <= off + half_step(np.abs(y) + off, out_type)), (np.abs(got - y) / (off + half_step(y, out_type))).max()
    assert bool((out[:, N:] == 77).all())


SIZES = [(1, 1), (16, 128), (17, 129), (70, 40), (200, 1000), (1500, 520)]


@pytest.mark.parametrize("N,K", SIZES)
@pytest.mark.parametrize("M", [1, 2, 16, 17, 40, 64, 65, 130])
def test_linear(M, N, K):
    rng = np.random.default_rng(M * 1000 + N + K)
    for i, dtype in enumerate(TYPES):
        w = Weights(rng, N, K, (32, 64, 128)[(M + i) % 3], ("f16", "bf16")[(M + N + i) % 2], zeros=(N + i) % 2 == 1)
        check_linear(rng, M, w, dtype, TYPES[(i + M) % 3], bias=i != 1, add=(None, "own", "in place")[(i + K) % 3], pitch=(0, 3, 8)[(i + N) % 3])


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(12, 512, 2500), (33, 300, 4100), (5, 2000, 640), (200, 530, 700)])
def test_linear_of_every_type_and_group(M, N, K, dtype, zeros, group):
    rng = np.random.default_rng(K + group)
    check_linear(rng, M, Weights(rng, N, K, group, "bf16" if zeros else "f16", zeros), dtype, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 64, 16000), (16, 100, 7000), (32, 33, 16384), (40, 200, 4500), (130, 70, 3333), (300, 64, 5000)])
def test_few_outputs_of_many_inputs(M, N, K, dtype):
    """The inputs are split among workgroups and their sums added up by another launch."""
    rng = np.random.default_rng(M + K)
    for i, group in enumerate((32, 128)):
        w = Weights(rng, N, K, group, zeros=i == 0)
        check_linear(rng, M, w, dtype, ("f32", dtype)[i], bias=i == 0, add=("in place", None)[i], pitch=3 * i)
    check_gated(rng, M, N, K, 64, dtype, "gelu")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(33, 17000, 2100), (64, 9000, 4200), (129, 700, 900), (257, 300, 260)])
def test_matrices_of_every_launch(M, N, K, dtype):
    """64 rows and 128 rows a workgroup, of matrices that are large enough, and of any with more rows."""
    rng = np.random.default_rng(M + K)
    for i, group in enumerate((32, 128)):
        check_linear(rng, M, Weights(rng, N, K, group, ("f16", "bf16")[i], zeros=i == 1), dtype, dtype)


@pytest.mark.parametrize("M,N,K", [(25, 64, 6272), (40, 100, 6400), (64, 17000, 2176), (129, 700, 128), (300, 270, 1024)])
def test_rows_from_where_they_lie(M, N, K):
    """fp16: rows with a pitch of whole 16 bytes, with another one, and from an address between, have the same results bit for bit."""
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(M + K)
    w = Weights(rng, N, K, 64, zeros=True)
    check_linear(rng, M, w, "f16", "f16", pitch=8)
    x = on_gpu(rows_of(rng, M, K, "f16"), "f16")
    ws, outs = workspace(binding.packed_workspace_bytes(w.pp, M)), []
    for pitch, begin in ((0, 0), (24, 8), (3, 0), (8, 1)):
        held = torch.full((M, K + pitch), float("nan"), dtype=torch.float16, device="cuda")
        held[:, begin:begin + K] = x
        outs.append(torch.empty(M, N, device="cuda"))
        binding.packed_linear(w.pp, w.on_gpu, held[:, begin:begin + K], ws, outs[-1])
    assert all(torch.equal(outs[0], out) for out in outs[1:])


def test_linear_results_do_not_depend_on_the_run():
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(8)
    w = Weights(rng, 900, 1100, 64, zeros=True)
    for M in (7, 90):
        x = on_gpu(rows_of(rng, M, 1100, "bf16"), "bf16")
        ws = workspace(binding.packed_workspace_bytes(w.pp, M))
        outs = [torch.empty(M, 900, dtype=torch.float32, device="cuda") for _ in range(3)]
        for out in outs:
            ws.random_(0, 255)
            binding.packed_linear(w.pp, w.on_gpu, x, ws, out)
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [3, 50, 140])
def test_rows_that_are_not_finite_are_alone(M, dtype):
    """A NaN or an infinity in a row reaches no other row; zeros of the row's results with it are no numbers either."""
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(M)
    w = Weights(rng, 150, 300, 32, zeros=True)
    x = rows_of(rng, M, 300, dtype)
    ws, out = workspace(binding.packed_workspace_bytes(w.pp, M)), [torch.empty(M, 150, dtype=torch.float32, device="cuda") for _ in range(2)]
    binding.packed_linear(w.pp, w.on_gpu, on_gpu(x, dtype), ws, out[0])
    x[1, 7], x[M - 1, 299] = np.nan, np.inf
    binding.packed_linear(w.pp, w.on_gpu, on_gpu(x, dtype), ws, out[1])
    good = [m for m in range(M) if m not in (1, M - 1)]
    assert torch.equal(out[0][good], out[1][good])
    assert not bool(torch.isfinite(out[1][[1, M - 1]]).any())


# ---- gated --------------------------------------------------------------------------------------

def check_gated(rng, M, N, K, group, dtype, act, out_type=None, zeros=(False, False), scale="f16"):
    """Tolerance: act has a slope of 1.13 at most; its own steps round some 8 times by 2^-23, of the value, or -- through the argument of e^x
    and erfc -- of 1."""
    import torch
    from paper_1806_00588_amd import binding
    gate, up = (Weights(rng, N, K, group, scale, z) for z in zeros)
    out_type = out_type or dtype
    x = rows_of(rng, M, K, dtype)
    (g, g_off), (u, u_off) = gate.product(x), up.product(x)
    a = layers.activation(g, act)
    a_off = 1.13 * g_off + 2.0 ** -20 * np.abs(a) + 2.0 ** -22
    want, off = a * u, a_off * (np.abs(u) + u_off) + np.abs(a) * u_off
    out = torch.empty(M, N, dtype=torch_type(out_type), device="cuda")
    ws = workspace(binding.packed_workspace_bytes(gate.pp, M))
    binding.packed_gated(gate.pp, gate.on_gpu, up.on_gpu, on_gpu(x, dtype), ws, out, act=act)
    got = in_64(out)
    assert np.all(np.abs(got - want) <= off + half_step(np.abs(want) + off, out_type)), (np.abs(got - want) / (off + half_step(want, out_type))).max()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("M,N,K", [(1, 16, 128), (1, 70, 33), (12, 1000, 200), (33, 130, 2100), (64, 2100, 129), (150, 211, 500)])
def test_gated(M, N, K, act):
    rng = np.random.default_rng(M + N + K)
    for i, dtype in enumerate(TYPES):
        check_gated(rng, M, N, K, (32, 64, 128)[(i + M) % 3], dtype, act, (None, "f32", "bf16")[(i + N) % 3], ((False, False), (True, True), (True, False))[(i + K) % 3],
                    ("f16", "bf16")[(i + N) % 2])


# ---- where a call runs --------------------------------------------------------------------------

def test_on_another_stream_and_in_a_graph():
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(5)
    w, up = Weights(rng, 400, 500, 64), Weights(rng, 400, 500, 64)
    ws = workspace(binding.packed_workspace_bytes(w.pp, 20))
    x = [on_gpu(rows_of(rng, 20, 500, "f16"), "f16") for _ in range(3)]
    held, out, both = torch.empty_like(x[0]), torch.empty(20, 400, dtype=torch.float16, device="cuda"), torch.empty(20, 400, dtype=torch.float16, device="cuda")

    def step():
        binding.packed_linear(w.pp, w.on_gpu, held, ws, out)
        binding.packed_gated(w.pp, w.on_gpu, up.on_gpu, held, ws, both, act="gelu")

    want = []
    for i in x:
        held.copy_(i)
        step()
        want.append((out.clone(), both.clone()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        held.copy_(x[0])
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want[0][0]) and torch.equal(both, want[0][1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(6):
        held.copy_(x[turn % 3])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[turn % 3][0]) and torch.equal(both, want[turn % 3][1])


def test_binding_refuses():
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(1)
    w = Weights(rng, 40, 100, 32)
    ws, x, out = workspace(256), torch.zeros(3, 100, device="cuda"), torch.zeros(3, 40, device="cuda")
    other = binding.packed_params(40, 101, 32)
    for call in (lambda: binding.packed_linear(other, w.on_gpu, torch.zeros(3, 101, device="cuda"), ws, out),
                 lambda: binding.packed_linear(w.pp, w.on_gpu, x[:, :99], ws, out),
                 lambda: binding.packed_linear(w.pp, w.on_gpu, x.t().contiguous().t(), ws, out),
                 lambda: binding.packed_linear(w.pp, w.on_gpu, x.cpu(), ws, out),
                 lambda: binding.packed_linear(w.pp, w.on_gpu, x.double(), ws, out),
                 lambda: binding.packed_linear(w.pp, w.on_gpu, x, ws, out, add=out.half()),
                 lambda: binding.packed_linear(w.pp, w.on_gpu, x, ws, out, bias=torch.zeros(39, device="cuda")),
                 lambda: binding.packed_gated(w.pp, w.on_gpu, w.on_gpu, x, ws, out, act="relu"),
                 lambda: binding.PackedWeights(w.pp, scales=torch.zeros(3, 1, 16, 1, dtype=torch.float16, device="cuda")),
                 lambda: binding.PackedWeights(w.pp, scales=torch.zeros(3, 1, 16, 4, device="cuda"))):
        with pytest.raises(ValueError):
            call()
