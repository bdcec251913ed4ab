"""The operators around a decoder with a cache together, as a search uses them: selection -> beam bookkeeping -> block tables -> keys and
values into the cache -> attention -> the next step's hidden rows, each step against the references on the same inputs, with the
selection from the caller's logits and with the decode step; and the loop as one HIP graph.  The model is a stand-in: queries,
keys and values of a word are looked up."""
import numpy as np
import pytest

import oracle.decoder as plain
import workloads
from gpu_harness import GpuCase, assert_topb_matches, to_dev
from oracle import beam as obeam
from test_gpu_beam_select import check as check_select
from test_gpu_cache import ROUNDING, assert_same_pool, from_pool

pytestmark = pytest.mark.gpu


class Search:
    """Device state of a search of S sentences of B beams over the tiny vocabulary, two layers of cache."""

    def __init__(self, S=2, B=4, steps=40, block=16, prompt=21, dtype="float32"):
        import torch
        import paper_1806_00588_amd as lsh
        from paper_1806_00588_amd import binding
        self.lsh, self.binding, self.torch = lsh, binding, torch
        cfg = workloads.CONFIGS["tiny"]
        self.gc = GpuCase.from_config(cfg)
        self.S, self.B, self.steps, self.prompt, self.block = S, B, steps, prompt, block
        R, self.V, d = S * B, cfg.V, cfg.d
        self.R, self.Hq, self.H, self.D = R, 4, 2, 16
        rng = np.random.default_rng(4)
        kind = getattr(torch, dtype)
        self.emb = [to_dev(rng.standard_normal((self.V, n, self.D)).astype(np.float32)).to(kind) for n in (self.Hq, self.H, self.H)]
        width = (prompt + steps) // block + 2
        self.cp = binding.cache_params(S, B, R * width + 7, block, width, self.H, self.D)
        self.pools = [binding.CachePool(self.cp) for _ in range(2)]
        self.ap = binding.attention_params(1, self.Hq, 0.25)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.tables = [torch.full((R, width), -1, **i32) for _ in range(2)]
        self.lengths = [torch.zeros(R, **i32) for _ in range(2)]
        self.slots, self.copy_from = torch.empty(R, 1, **i32), torch.empty(R, **i32)
        self.shared, self.status = torch.empty(S, **i32), torch.empty(2, **i32)
        self.cache_ws = self.room(binding.cache_workspace_bytes(self.cp))
        self.attn_ws = self.room(binding.attention_workspace_bytes(self.cp, self.ap))
        self.q = torch.empty(R, 1, self.Hq, self.D, dtype=kind, device="cuda")
        self.out = torch.zeros_like(self.q)
        self.hidden = torch.empty(R, d, device="cuda")
        self.hist = binding.BeamHistory(S, B, steps, eos=3)
        self.beam, self.word = torch.zeros(R, **i32), torch.zeros(R, **i32)
        self.score, self.scores = torch.empty(R, device="cuda"), torch.zeros(R, device="cuda")
        self.sp, self.ssp = binding.step_params(S, B, cfg.T), binding.select_params(S, B, self.V)
        self.step_ws = self.room(lsh.step_workspace_bytes(self.gc.tables, self.sp))
        self.select_ws = self.room(binding.select_workspace_bytes(self.ssp))
        self.prompts = to_dev(rng.integers(0, self.V, (R, prompt)).astype(np.int64))
        self.n_prompt = to_dev(np.where(np.arange(R) % B == 0, prompt - np.arange(R) // B, 0).astype(np.int32))

    def room(self, n):
        return self.torch.empty(n, dtype=self.torch.uint8, device="cuda")

    def begin(self):
        """The prompts into row 0 of each sentence; one living beam."""
        t, b = self.torch, self.binding
        slots = t.empty(self.R, self.prompt, dtype=t.int32, device="cuda")
        for x in self.lengths:
            x.zero_()
        b.cache_advance(self.cp, self.prompt, self.tables[1], self.lengths[1], self.tables[0], self.lengths[0], slots, self.copy_from,
                        self.shared, self.status, self.cache_ws, n_new=self.n_prompt)
        for layer, pool in enumerate(self.pools):
            b.cache_write(self.cp, pool, self.emb[1][self.prompts + 0 * layer], self.emb[2][self.prompts], slots, self.copy_from)
        self.out.zero_()
        self.scores.zero_()
        self.scores.view(self.S, self.B)[:, 1:] = -float("inf")
        self.hidden.copy_(self.emb[0][self.prompts[:, 0]].reshape(self.R, -1).float())

    def choose(self, step, logits):
        """A selection and its bookkeeping; logits None: by the decode step."""
        b = self.binding
        if logits is None:
            self.lsh.decode_step(self.gc.tables, self.hidden, self.scores, self.gc.topfreq_dev, self.sp, self.step_ws, self.beam, self.word, self.score)
        else:
            b.beam_select(self.ssp, logits, self.scores, self.select_ws, self.beam, self.word, self.score)
        b.beam_advance(self.hist, step, self.beam, self.word, self.score, [], [], self.scores)

    def cache_step(self, step):
        """Tables after the choice, the chosen words' keys and values, attention in both layers, the next hidden rows."""
        t, b = self.torch, self.binding
        i, o = step & 1, (step + 1) & 1
        b.cache_advance(self.cp, 1, self.tables[i], self.lengths[i], self.tables[o], self.lengths[o], self.slots, self.copy_from, self.shared,
                        self.status, self.cache_ws, parents=self.beam)
        words = self.word.clamp(min=0)
        k, v = self.emb[1].index_select(0, words), self.emb[2].index_select(0, words)
        self.q.copy_(self.emb[0].index_select(0, words).unsqueeze(1))
        for layer, pool in enumerate(self.pools):
            b.cache_write(self.cp, pool, k.unsqueeze(1), v.unsqueeze(1), self.slots, self.copy_from)
            b.cache_attention(self.cp, self.ap, pool, self.q, self.tables[o], self.lengths[o], self.attn_ws, self.out, shared=self.shared)
            self.q.add_(self.out)
        self.hidden.copy_(self.q.view(self.R, -1))


def host(x):
    return x.double().cpu().numpy() if x.is_floating_point() else x.cpu().numpy()


@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_every_step_of_a_search(dense, dtype):
    import torch
    s = Search(dtype=dtype)
    s.begin()
    torch.cuda.synchronize()
    S, B, R = s.S, s.B, s.R
    ref = [from_pool(p) for p in s.pools]
    tables, lengths = host(s.tables[0]), host(s.lengths[0])
    inside, last = ROUNDING["f32" if dtype == "float32" else "bf16"]
    for step in range(s.steps):
        scores, hidden = s.scores.cpu().numpy().copy(), s.hidden.cpu().numpy()
        logits = s.hidden @ s.gc.E_dev.t() if dense else None
        s.choose(step, logits)
        torch.cuda.synchronize()
        beam, word, score = (x.cpu().numpy().reshape(S, B) for x in (s.beam, s.word, s.score))
        if dense:
            check_select((beam, word, score, host(torch.logsumexp(logits.double(), 1)).astype(np.float32)), host(logits), scores, S, B, B)
        for n in range(S):
            rows = slice(n * B, n * B + B)
            if not dense:
                want = s.gc.oracle_sentence(hidden[rows], scores[rows], B)
                assert_topb_matches(beam[n], word[n], score[n], want, scores[rows])
            assert np.array_equal(s.scores.cpu().numpy()[rows], obeam.advance(beam[n], word[n], score[n], [], 3)[1])
        s.cache_step(step)
        torch.cuda.synchronize()
        o = (step + 1) & 1
        want = plain.advance(S, B, 1, s.cp.n_blocks, s.block, tables, lengths, beam.reshape(-1))
        for name, got in (("tables", s.tables[o]), ("lengths", s.lengths[o]), ("slots", s.slots), ("copy_from", s.copy_from),
                          ("shared", s.shared), ("status", s.status)):
            assert np.array_equal(host(got).reshape(want[name].shape), want[name]), (step, name)
        assert want["status"].tolist() == [0, 0]
        tables, lengths = want["tables"], want["lengths"]
        words = np.maximum(word.reshape(-1), 0)
        k, v = host(s.emb[1])[words][:, None], host(s.emb[2])[words][:, None]
        q = s.emb[0][torch.from_numpy(words).cuda()].unsqueeze(1)
        for layer in range(2):
            plain.write(ref[layer], k, v, want["slots"], want["copy_from"])
            got = from_pool(s.pools[layer])
            for r in range(R):                      # (blocks that nobody has hold what they held)
                ids = tables[r, :-(-lengths[r] // s.block)]
                assert_same_pool(plain.Pool(got.k[ids], got.v[ids], got.k_scale[ids], got.v_scale[ids]),
                                 plain.Pool(ref[layer].k[ids], ref[layer].v[ids], ref[layer].k_scale[ids], ref[layer].v_scale[ids]))
            out, _, size, reach = plain.attention(ref[layer], host(q), tables, lengths, 0.25)
            if layer == 0:                          # the second layer's queries, from the first's result as the device rounds it
                first = torch.empty_like(s.out)
                s.binding.cache_attention(s.cp, s.ap, s.pools[0], q, s.tables[o], s.lengths[o], s.attn_ws, first, shared=s.shared)
                got_out = first
                q = q + first
            else:
                got_out = s.out
            off = 2 * (s.D + 2) * 2.0 ** -24 * reach + 2.0 ** -20 + int(max(lengths)) * 2.0 ** -24 + inside
            assert np.all(np.abs(host(got_out) - out) <= off[..., None] * size + last * np.abs(out) + 1e-30), (step, layer)
    assert lengths.max() > 3 * s.block and int(want["shared"].max()) > 0


def test_the_loop_as_one_graph():
    import torch
    s = Search(steps=9, dtype="bfloat16")

    def loop():
        s.begin()
        for step in range(s.steps):
            s.choose(step, None)
            s.cache_step(step)

    loop()
    torch.cuda.synchronize()
    outs = lambda: [x.cpu().clone() for x in (s.out, s.scores, s.hist.backptr, s.hist.words, s.hist.scores, s.tables[1], s.lengths[1], s.shared)]   # noqa: E731
    want = outs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loop()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        loop()
    for k in range(4):
        s.out.fill_(5.0)
        s.cache_ws.fill_(k * 60), s.attn_ws.fill_(k * 60), s.step_ws.fill_(k * 60)
        for pool in s.pools:                         # what blocks held before does not matter
            pool.k.fill_(127), pool.v.fill_(255), pool.k_scale.fill_(float("nan")), pool.v_scale.fill_(float("inf"))
        if k == 2:
            loop()                                   # the program's own work between replays
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, outs()):
            assert torch.equal(a, b)
