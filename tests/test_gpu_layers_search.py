"""A beam search with a decoder whose layers keep a recurrent state, made of the calls for it: projections of 4 bits, the gated delta rule from the parents'
states, a gated block, the output layer, the selection.  Every result is compared with the reference of its operator on the very inputs that it got (by
the tolerances of those operators' own tests), and the steps replayed as a graph with the steps called one by one."""
import numpy as np
import pytest

from oracle import layers
from test_gpu_packed import Weights, half_step, in_64, on_gpu, workspace

pytestmark = pytest.mark.gpu

S, B, D, HEADS, K_HEADS, DK, DV, FF, V = 3, 4, 160, 4, 2, 32, 48, 300, 531
R, WIDE = S * B, 2 * K_HEADS * DK + HEADS * DV


class Decoder:
    """One layer, its buffers for T tokens of a row, bf16 throughout but the logits."""

    def __init__(self, T):
        import torch
        from paper_1806_00588_amd import binding
        rng = np.random.default_rng(4)
        self.lib, self.T = binding, T
        self.qkv, self.gates = Weights(rng, WIDE, D, 64), Weights(rng, 2 * HEADS, D, 32, "bf16", True)
        self.out, self.gate, self.up = Weights(rng, D, HEADS * DV, 32, zeros=True), Weights(rng, FF, D, 128), Weights(rng, FF, D, 128)
        self.down, self.words = Weights(rng, D, FF, 64, "bf16"), Weights(rng, V, D, 32, "bf16", True)
        bf16 = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")
        f32 = lambda *shape: torch.zeros(*shape, device="cuda")
        M = R * T
        self.row, self.raw, self.mixed, self.x1, self.h, self.x2 = bf16(M, WIDE), f32(M, 2 * HEADS), bf16(R, T, HEADS, DV), bf16(M, D), bf16(M, FF), bf16(M, D)
        self.decay, self.beta, self.logits = f32(R, T, HEADS), f32(R, T, HEADS), f32(R, V)
        self.dp = binding.delta_params(S, B, T, HEADS, K_HEADS, DK, DV, DK ** -0.5)
        self.ws = workspace(max([binding.packed_workspace_bytes(w.pp, M) for w in (self.qkv, self.gates, self.out, self.gate, self.down, self.words)] +
                                [binding.delta_workspace_bytes(self.dp)]))

    def parts(self):
        row = self.row.view(R, self.T, WIDE)
        return [x.unflatten(2, (heads, -1)) for x, heads in zip(row.split([K_HEADS * DK, K_HEADS * DK, HEADS * DV], 2), (K_HEADS, K_HEADS, HEADS))]

    def run(self, x, state_in, state_out, parents, n_new=None):
        """x [R * T, D] -> x2; torch makes what lies between the calls."""
        import torch
        lib, M = self.lib, R * self.T
        lib.packed_linear(self.qkv.pp, self.qkv.on_gpu, x, self.ws, self.row)
        lib.packed_linear(self.gates.pp, self.gates.on_gpu, x, self.ws, self.raw)
        for t in self.parts()[:2]:                 # queries and keys of length 1, in place
            t.copy_(torch.nn.functional.normalize(t.float(), dim=-1))
        raw = self.raw.view(R, self.T, 2, HEADS)
        self.decay.copy_(-torch.nn.functional.softplus(raw[:, :, 0]))
        self.beta.copy_(torch.sigmoid(raw[:, :, 1]))
        q, k, v = self.parts()
        lib.delta_rule(self.dp, q, k, v, self.decay, self.beta, state_in, state_out, self.ws, self.mixed, parents=parents, n_new=n_new)
        lib.packed_linear(self.out.pp, self.out.on_gpu, self.mixed.view(M, HEADS * DV), self.ws, self.x1, add=x)
        lib.packed_gated(self.gate.pp, self.gate.on_gpu, self.up.on_gpu, self.x1, self.ws, self.h, act="silu")
        self.x2.copy_(self.x1)
        lib.packed_linear(self.down.pp, self.down.on_gpu, self.h, self.ws, self.x2, add=self.x2)

    def check(self, x, state_in, state_out, parents, n_new=None):
        """What the last run left, operator by operator."""
        def near(got, want, off, dtype):
            got = in_64(got)
            assert np.all(np.abs(got - want) <= off + half_step(np.abs(want) + off, dtype)), (np.abs(got - want) / (off + half_step(want, dtype))).max()

        def product(w, x, got, dtype, add=None):
            y, off = w.product(in_64(x))
            if add is not None:
                y, off = y + in_64(add), off + (w.group + 12) * 2.0 ** -23 * np.abs(in_64(add))
            near(got, y, off, dtype)

        M = R * self.T
        q, k, v = (in_64(t) for t in self.parts())
        begin = in_64(state_in)
        begin = np.stack([begin[r // B * B + p] for r, p in enumerate(parents.tolist())])
        n = np.full(R, self.T) if n_new is None else n_new.cpu().numpy()
        want, after, size = layers.delta_rule(q, k, v, in_64(self.decay), in_64(self.beta), begin, DK ** -0.5, n)
        # (keys rounded to bf16 are up to 2^-8 longer than 1: what a token adds to may grow by twice that)
        tol = (1 + 2.0 ** -7) ** self.T * 2.0 ** -24 * 16 * np.sqrt((n + 1) * (DK + 64))[:, None, None] * size
        assert np.all(np.abs(in_64(state_out) - after) <= tol[:, :, None])
        for r in range(R):
            near(self.mixed[r, :n[r]], want[r, :n[r]], np.broadcast_to(tol[r] * DK ** -0.5 * (1 + 2.0 ** -8), want[r, :n[r]].shape), "bf16")
        product(self.gates, x, self.raw, "f32")
        product(self.out, self.mixed.view(M, HEADS * DV), self.x1, "bf16", x)
        (g, g_off), (u, u_off) = self.gate.product(in_64(self.x1)), self.up.product(in_64(self.x1))
        a = layers.activation(g, "silu")
        near(self.h, a * u, (1.13 * g_off + 2.0 ** -20 * np.abs(a) + 2.0 ** -22) * (np.abs(u) + u_off) + np.abs(a) * u_off, "bf16")
        product(self.down, self.h, self.x2, "bf16", self.x1)


def test_a_search_step_by_step_and_as_a_graph():
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(9)
    embed = on_gpu(rng.normal(size=(V, D)), "bf16")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    # prompts: the first beam of each sentence has 70, 1 and 37 tokens; the others none
    T = 70
    prompt = Decoder(T)
    x = embed[torch.from_numpy(rng.integers(0, V, R * T)).cuda()]
    n_new = i32([n if b == 0 else 0 for n in (70, 1, 37) for b in range(B)])
    states = [torch.zeros(R, HEADS, DK, DV, device="cuda") for _ in range(2)]
    itself = i32(list(range(B)) * S)
    prompt.run(x, states[0], states[1], itself, n_new)
    prompt.check(x, states[0], states[1], itself, n_new)
    # steps: all beams begin with the first one's state, then with their parents'
    step, sp = Decoder(1), binding.select_params(S, B, V)
    ws = workspace(binding.select_workspace_bytes(sp))
    beam, word = (torch.zeros(R, dtype=torch.int32, device="cuda") for _ in range(2))
    score, new_score, begin_score = torch.zeros(R, device="cuda"), torch.zeros(R, device="cuda"), on_gpu(np.tile([0.0] + [-np.inf] * (B - 1), S).astype(np.float32))
    first_word = on_gpu(rng.integers(0, V, R).astype(np.float32)).to(torch.int32)
    x1, seen = torch.empty(R, D, dtype=torch.bfloat16, device="cuda"), []

    def one(i):
        x1.copy_(embed[word.long()])
        step.run(x1, states[1 - i % 2], states[i % 2], beam)
        binding.packed_linear(step.words.pp, step.words.on_gpu, step.x2, step.ws, step.logits)
        binding.beam_select(sp, step.logits, score, ws, beam, word, new_score)
        score.copy_(new_score)

    def start():
        states[1].copy_(after_prompt)
        beam.zero_()
        word.copy_(first_word)
        score.copy_(begin_score)

    after_prompt = states[1].clone()
    start()
    for i in range(6):
        parents = beam.clone()
        one(i)
        step.check(x1, states[1 - i % 2], states[i % 2], parents)
        y, off = step.words.product(in_64(step.x2))
        assert np.all(np.abs(in_64(step.logits) - y) <= off + half_step(np.abs(y) + off, "f32"))
        assert bool((beam >= 0).all()) and bool(torch.isfinite(score).all())
        seen.append((beam.clone(), word.clone(), score.clone(), states[i % 2].clone()))
    assert any(len(set(b[s * B:(s + 1) * B].tolist())) < B for b, *_ in seen for s in range(S))      # (beams that share a parent are among them)
    start()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(0)
        one(1)
    for turn in range(3):
        start()
        for i in range(0, 6, 2):
            graph.replay()
            torch.cuda.synchronize()
            for got, want in zip((beam, word, score, states[1]), seen[i + 1]):
                assert torch.equal(got, want)
