"""lsh_cache_advance against oracle/decoder.py: whole numbers, equal."""
import numpy as np
import pytest

import oracle.decoder as plain
from gpu_harness import to_dev

pytestmark = pytest.mark.gpu
NAMES = ("tables", "lengths", "slots", "copy_from", "shared", "status")


def call(cp, T, tables, lengths, parents=None, n_new=None, shared=True, stream=None):
    """One call on device tensors; returns device tensors by name."""
    import torch
    from paper_1806_00588_amd import binding
    R = cp.S * cp.B
    out = {k: torch.full(shape, -77, dtype=torch.int32, device="cuda") for k, shape in
           zip(NAMES, ((R, cp.max_blocks), (R,), (R, T), (R,), (cp.S,), (2,)))}
    ws = torch.full((binding.cache_workspace_bytes(cp),), 255, dtype=torch.uint8, device="cuda")
    binding.cache_advance(cp, T, tables, lengths, out["tables"], out["lengths"], out["slots"], out["copy_from"], out["shared"] if shared else None,
                          out["status"], ws, parents=parents, n_new=n_new, stream=stream)
    return out


def ints(x):
    return None if x is None else to_dev(np.ascontiguousarray(x, dtype=np.int32))


def check(S, B, T, n_blocks, block, tables, lengths, parents=None, n_new=None):
    import torch
    from paper_1806_00588_amd import binding
    cp = binding.cache_params(S, B, n_blocks, block, tables.shape[1], 1, 16)
    got = call(cp, T, ints(tables), ints(lengths), ints(parents), ints(n_new))
    torch.cuda.synchronize()
    want = plain.advance(S, B, T, n_blocks, block, tables, lengths, parents, n_new)
    for k in NAMES:
        assert np.array_equal(got[k].cpu().numpy(), want[k]), k
    return want


def rows(rng, S, B, block, width, longest, common, n_blocks):
    """Tables of S * B rows, `common` tokens of each sentence's shared, blocks in random places."""
    ids = iter(rng.permutation(n_blocks).tolist())
    tables, lengths = rng.integers(-5, n_blocks + 5, (S * B, width)), np.zeros(S * B, dtype=int)   # (what is behind a row is not read)
    for s in range(S):
        head = [next(ids) for _ in range(common // block)]
        for b in range(B):
            n = int(rng.integers(common, longest + 1))
            t = head + [next(ids) for _ in range(-(-n // block) - len(head))]
            tables[s * B + b, :len(t)], lengths[s * B + b] = t, n
    return tables, lengths


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("S,B,width,longest,common,T", [(1, 1, 4, 60, 0, 1), (1, 12, 12, 150, 64, 1), (5, 3, 20, 250, 128, 1), (2, 7, 9, 120, 16, 40),
                                                       (3, 20, 40, 600, 0, 3), (40, 4, 30, 300, 256, 1), (1, 256, 6, 80, 16, 2)])
def test_matches_plain(S, B, width, longest, common, T, block):
    rng = np.random.default_rng(block + S * B)
    longest, common = min(longest, width * block - T), common // block * block
    longest = max(longest, common)
    n_blocks = S * B * width + 5
    tables, lengths = rows(rng, S, B, block, width, longest, common, n_blocks)
    parents, n_new = rng.integers(-1, B, S * B), rng.integers(0, T + 1, S * B)
    for p, n in ((None, None), (parents, None), (None, n_new), (parents, n_new), (np.zeros(S * B, dtype=int), None)):
        check(S, B, T, n_blocks, block, tables, lengths, p, n)


@pytest.mark.parametrize("S,B,width,longest,common,T", [(3, 5, 2500, 700, 320, 1), (40, 10, 90, 1300, 800, 2), (1200, 1, 5, 60, 0, 3), (5, 250, 30, 300, 128, 1),
                                                       (64, 10, 258, 4100, 3600, 1), (2, 2, 9000, 140000, 100000, 40)])
def test_matches_plain_beyond_one_workgroup(S, B, width, longest, common, T):
    """More rows, more entries or more blocks than one workgroup takes."""
    rng = np.random.default_rng(width)
    block = 16
    n_blocks = int(S * (common // block + B * ((longest - common) // block + 3))) + 70
    tables, lengths = rows(rng, S, B, block, width, longest, common, n_blocks)
    parents, n_new = rng.integers(-1, B, S * B), rng.integers(0, T + 1, S * B)
    for p, n in ((None, None), (parents, n_new)):
        check(S, B, T, n_blocks, block, tables, lengths, p, n)


def test_lengths_of_zero_one_and_whole_blocks():
    tables = np.array([[3, 9], [5, 9], [1, 0], [4, 6], [9, 9], [2, 9]])
    for lengths in ([0, 1, 32, 17, 0, 16], [0] * 6, [16, 16, 32, 31, 0, 15]):
        for T in (1, 16):
            if max(lengths) + T <= 48:
                check(2, 3, T, 30, 16, np.hstack([tables, np.full((6, 1), -1)]), np.array(lengths), None, None)


def test_a_search_from_its_prompt_to_its_end():
    """Many steps by the operator alone: the prompt in row 0, then all beams from it, then random parents.  No two rows ever write on a block
    that both have, and every row's history is its parents'."""
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(5)
    S, B, block, width, n_blocks = 3, 6, 16, 12, 150
    cp = binding.cache_params(S, B, n_blocks, block, width, 1, 16)
    R = S * B
    tables, lengths = np.full((R, width), -1), np.zeros(R, dtype=int)
    history = [[] for _ in range(R)]            # what each row's tokens are
    cells, serial = {}, 0                       # slot: token
    for step in range(100):
        T = 50 if step == 0 else 1
        if step == 0:
            parents, n_new = None, np.where(np.arange(R) % B == 0, rng.integers(30, 51, R), 0)
        else:
            parents = np.zeros(R, dtype=int) if step == 1 else np.where(rng.random(R) < 0.1, -1, rng.integers(0, B, R))
            for s in range(S):                  # a living row for each sentence
                live = [b for b in range(B) if lengths[s * B + b] > 0]
                at = slice(s * B, s * B + B)
                parents[at] = [int(rng.choice(live)) if p < 0 or p not in live else int(p) for p in parents[at]]
            parents[rng.integers(R)] = -1
            n_new = None
        dev = call(cp, T, ints(tables), ints(lengths), ints(parents), ints(n_new))
        torch.cuda.synchronize()
        got = {k: v.cpu().numpy() for k, v in dev.items()}
        want = plain.advance(S, B, T, n_blocks, block, tables, lengths, parents, n_new)
        assert all(np.array_equal(got[k], want[k]) for k in NAMES), step
        assert np.all(got["status"] == 0)
        old, new = dict(cells), []
        for r in range(R):
            p = r if parents is None else (r - r % B + parents[r] if parents[r] >= 0 else -1)
            h = list(history[p]) if p >= 0 else []
            mine = got["slots"][r][got["slots"][r] >= 0]
            if got["copy_from"][r] >= 0:
                for i in range(len(h) % block):
                    cells[int(mine[0]) // block * block + i] = old[int(got["copy_from"][r]) * block + i]
            for m in mine:
                cells[int(m)] = serial
                h.append(serial)
                serial += 1
            new.append(h)
        history, tables, lengths = new, got["tables"], got["lengths"]
        for r in range(R):
            assert lengths[r] == len(history[r])
            assert [cells[int(tables[r, i // block]) * block + i % block] for i in range(len(history[r]))] == history[r]
        if max(lengths) + 1 > width * block:
            break
    assert step > 60


def test_not_enough_blocks_and_too_long_rows():
    rng = np.random.default_rng(6)
    tables, lengths = rows(rng, 2, 4, 16, 8, 100, 32, 64)
    used = len({int(i) for r in range(8) for i in tables[r, :-(-lengths[r] // 16)]})
    for spare in (0, 1, 3):                     # as many blocks as are in use, and a few more: ids have to stay inside
        ids = {int(i): k for k, i in enumerate(sorted({int(i) for r in range(8) for i in tables[r, :-(-lengths[r] // 16)]}))}
        t = np.vectorize(lambda i: ids.get(int(i), -1))(tables)
        want = check(2, 4, 16, used + spare, 16, t, lengths, None, np.full(8, 16))
        assert want["status"][0] == 8 - spare and np.all(want["slots"] == -1)
    want = check(2, 4, 40, 200, 16, tables, np.minimum(lengths, 90), None, np.array([0, 40, 1, 39, 5, 40, 40, 38]))
    assert want["status"][1] > 0 and np.all(want["copy_from"] == -1)


def test_every_free_block_and_not_one_more():
    """Prompts that take all blocks of a pool, in one call; and more rows than a workgroup has threads."""
    for S, block, T in ((1, 16, 16 * 30), (1500, 16, 16), (3000, 32, 7), (1000, 16, 33), (33, 16, 15)):
        n = -(-T // block)
        check(S, 1, T, S * n, block, np.full((S, n), -1), np.zeros(S, dtype=int))
        assert check(S, 1, T, max(1, S * n - 1), block, np.full((S, n), -1), np.zeros(S, dtype=int))["status"][0] == 1


def test_large_pool():
    """Free blocks behind more than one sweep over the pool (16384 blocks at a time), in use but for a few at its end."""
    rng = np.random.default_rng(7)
    n_blocks, width = 60000, 2100
    ids = rng.permutation(n_blocks)[:56000].reshape(28, 2000)
    tables = np.full((28, width), -1)
    tables[:, :2000] = ids
    check(28, 1, 130, n_blocks, 16, tables, np.full(28, 32000), None, rng.integers(0, 131, 28))


@pytest.mark.parametrize("R,width,n_blocks,T", [(1024, 32, 1 << 17, 64), (1024, 32, (1 << 17) + 1, 64), (1024, 33, 1 << 17, 64), (1, 32768, 1 << 17, 65536)])
def test_the_largest_calls_of_one_workgroup(R, width, n_blocks, T):
    rng = np.random.default_rng(R)
    old = rng.integers(0, width * 16 - T + 1, R) if R > 1 else np.array([width * 16 - T])
    ids, at = rng.permutation(n_blocks), 0
    tables = np.full((R, width), -1)
    for r in range(R):
        n = -(-int(old[r]) // 16)
        tables[r, :n] = ids[at:at + n]
        at += n
    check(R, 1, T, n_blocks, 16, tables, old, None, rng.integers(0, T + 1, R))


def test_senseless_input_stays_inside():
    """Lengths below zero or beyond the table, blocks that no pool has, parents that no sentence has: nothing outside the arrays is
    touched, and what can be said is said."""
    import torch
    from paper_1806_00588_amd import binding
    cp = binding.cache_params(2, 3, 20, 16, 4, 1, 16)
    tables = np.array([[1, -5, 99, 1 << 30]] * 6)
    got = call(cp, 5, ints(tables), ints([-5, 1 << 30, 64, 20, 63, 0]), ints([0, 1, 7, -9, 1 << 30, 2]), ints([1, 2, 3, 5, -4, 9]))
    torch.cuda.synchronize()
    assert got["status"].tolist()[1] > 0 and torch.all(got["slots"] == -1)
    got = call(cp, 5, ints(tables), ints([20, 20, 40, 20, 20, 0]), None, ints([1, 2, 3, 5, -4, 5]))
    torch.cuda.synchronize()
    slots = got["slots"].cpu().numpy()
    assert got["status"].tolist() == [0, 0] and np.all(slots < 20 * 16) and np.all(slots >= -1)


def test_without_shared_and_as_a_graph():
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(8)
    S, B, block, width, n_blocks = 4, 5, 16, 10, 300
    tables, lengths = rows(rng, S, B, block, width, 120, 48, n_blocks)
    cp = binding.cache_params(S, B, n_blocks, block, width, 1, 16)
    parents = rng.integers(0, B, S * B)
    want = plain.advance(S, B, 1, n_blocks, block, tables, lengths, parents)
    t, n, p = ints(tables), ints(lengths), ints(parents)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = call(cp, 1, t, n, p, shared=False, stream=side)
    torch.cuda.synchronize()
    assert torch.all(got["shared"] == -77)
    assert all(np.array_equal(got[k].cpu().numpy(), want[k]) for k in NAMES if k != "shared")
    out = {k: torch.empty_like(v) for k, v in got.items()}
    ws = torch.empty(binding.cache_workspace_bytes(cp), dtype=torch.uint8, device="cuda")

    def step():
        binding.cache_advance(cp, 1, t, n, out["tables"], out["lengths"], out["slots"], out["copy_from"], out["shared"], out["status"], ws, parents=p)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for k in range(4):
        if k == 2:
            parents = rng.integers(-1, B, S * B)
            p.copy_(ints(parents))
            want = plain.advance(S, B, 1, n_blocks, block, tables, lengths, parents)
        for x in out.values():
            x.fill_(-3)
        ws.fill_(k * 85)
        g.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(out[key].cpu().numpy(), want[key]) for key in NAMES)


def test_binding_refuses():
    import torch
    from paper_1806_00588_amd import binding
    cp = binding.cache_params(2, 3, 20, 16, 4, 1, 16)
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")   # noqa: E731
    ok = dict(tables_in=z(6, 4), lengths_in=z(6), tables_out=z(6, 4), lengths_out=z(6), slots=z(6, 2), copy_from=z(6), shared=z(2), status=z(2),
              workspace=torch.empty(binding.cache_workspace_bytes(cp), dtype=torch.uint8, device="cuda"))
    for bad in ({"tables_in": z(6, 3)}, {"lengths_in": z(5)}, {"slots": z(6, 1)}, {"shared": z(1)}, {"status": z(3)}, {"parents": z(5)},
                {"n_new": z(7)}, {"tables_out": z(6, 4).long()}, {"lengths_in": z(6).cpu()}, {"tables_in": z(4, 6).t()}):
        with pytest.raises(ValueError):
            binding.cache_advance(cp, 2, **{**ok, **bad})
    with pytest.raises(binding.LshBeamError):
        binding.cache_advance(cp, 2, **{**ok, "tables_out": ok["tables_in"]})


@pytest.mark.parametrize("R,width,n_blocks,T", [(64, 64, 1 << 17, 32), (65, 63, 5000, 31), (64, 65, 5000, 32), (8, 512, 5000, 256), (7, 64, 5000, 257),
                                                (9, 64, 5000, 230), (1, 4096, 1 << 17, 1), (64, 64, (1 << 17) + 1, 32)])
def test_both_sides_of_the_border_of_one_workgroup(R, width, n_blocks, T):
    rng = np.random.default_rng(R + T)
    old = rng.integers(0, width * 16 - T + 1, R)
    ids, at = rng.permutation(n_blocks), 0
    tables = np.full((R, width), -1)
    for r in range(R):
        n = min(-(-int(old[r]) // 16), (n_blocks - at) // 2)
        old[r] = min(old[r], n * 16)
        tables[r, :n] = ids[at:at + n]
        at += n
    check(R, 1, T, n_blocks, 16, tables, old, None, rng.integers(0, T + 1, R))


def test_senseless_input_of_many_rows_stays_inside():
    """The same for calls of more rows than one workgroup takes."""
    import torch
    from paper_1806_00588_amd import binding
    cp = binding.cache_params(40, 3, 20, 16, 4, 1, 16)
    tables = np.array([[1, -5, 99, 1 << 30]] * 120)
    got = call(cp, 5, ints(tables), ints([-5, 1 << 30, 64, 20, 63, 0] * 20), ints([0, 1, 7, -9, 1 << 30, 2] * 20), ints([1, 2, 3, 5, -4, 9] * 20))
    torch.cuda.synchronize()
    assert got["status"].tolist()[1] > 0 and torch.all(got["slots"] == -1)
    got = call(cp, 5, ints(tables), ints([20, 20, 40, 20, 20, 0] * 20), None, ints([1, 2, 3, 5, -4, 5] * 20))
    torch.cuda.synchronize()
    slots = got["slots"].cpu().numpy()
    assert got["status"].tolist()[1] == 0 and np.all(slots < 20 * 16) and np.all(slots >= -1)
