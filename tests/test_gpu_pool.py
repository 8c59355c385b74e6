"""Block tables and token maps through the C ABI against a sequential model; whole numbers, equal."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    torch.cuda.set_device(0)
    return kvarn


class Model:
    """The pool as lists: one sequence after the other."""

    def __init__(self, batch, max_blocks, n_phys, sink):
        self.sink, self.max_blocks, self.n_phys = sink, max_blocks, n_phys
        self.free, self.rows, self.err = list(range(n_phys)), [[] for _ in range(batch)], 0

    def step(self, lengths, extra=0):
        need = []
        for row, n in zip(self.rows, lengths):
            k = len(row) if n < 0 else max(int(n) + extra - self.sink, 0) // 128
            if k > self.max_blocks:
                self.err |= 1
                k = len(row)
            need.append(k)
        for row, k in zip(self.rows, need):
            self.free += row[k:]
            del row[k:]
        for row, k in zip(self.rows, need):
            if k - len(row) > len(self.free):
                self.err |= 1
                break  # nothing behind it grows
            while len(row) < k:
                row.append(self.free.pop(0))
        else:
            return
        at = next(i for i, (row, k) in enumerate(zip(self.rows, need)) if k - len(row) > 0)
        assert all(len(row) <= k for row, k in zip(self.rows[at:], need[at:]))


def make(K, batch, max_blocks, n_phys, sink, n_kv=1):
    p = K.kvarn_params_init(2, n_sink=sink)
    cache = K.Cache(p, batch, n_kv, max_blocks, n_phys=n_phys)
    return p, cache, K.BlockPool(cache)


def same(cache, pool, model):
    torch.cuda.synchronize()
    n = pool.n_blocks.cpu().numpy()
    assert n.tolist() == [len(r) for r in model.rows]
    want = np.full((len(model.rows), model.max_blocks), -1)
    for i, r in enumerate(model.rows):
        want[i, :len(r)] = r
    assert np.array_equal(cache.block_table.cpu().numpy(), want)
    first, count, a, b = pool.ring.tolist()
    ids = pool.free_ids.cpu().numpy()
    assert count == len(model.free) and (a, b) == (0, 0)
    assert [int(ids[(first + i) % model.n_phys]) for i in range(count)] == model.free
    assert int(cache.err_word) == model.err


@pytest.mark.parametrize("batch", [1, 3, 64, 255, 512, 513, 1000, 1025, 2600])
@pytest.mark.parametrize("sink,tight", [(0, False), (100, True)])
def test_random_steps(K, batch, sink, tight):
    """Sequences grow, shrink, end and begin, in pools with room to spare and in tight ones, where blocks are handed on."""
    rng = np.random.default_rng(batch)
    max_blocks = 40
    p, cache, pool = make(K, batch, max_blocks, max(batch * (6 if tight else 40), 3), sink)
    model = Model(batch, max_blocks, cache.n_phys, sink)
    lengths = np.zeros(batch, np.int64)
    for step in range(12):
        for i in range(batch):
            r = rng.random()
            lengths[i] = (lengths[i] + rng.integers(0, 200) if r < 0.5 else 0 if r < 0.7 else -1 if r < 0.75 else
                          rng.integers(0, sink + 128 * 14))
            lengths[i] = min(lengths[i], sink + 128 * 40)
        extra = int(rng.integers(0, 3)) * 64
        K.kvarn_assign_blocks(p, cache, pool, torch.from_numpy(lengths.astype(np.int32)).cuda(), extra)
        model.step(lengths, extra)
        same(cache, pool, model)
        lengths = np.maximum(lengths, 0)


def test_lengths_of_the_cache(K):
    p, cache, pool = make(K, 5, 9, 30, 7)
    cache.seq_len.copy_(torch.tensor([0, 134, 135, 7 + 128 * 9, 500], dtype=torch.int32))
    K.kvarn_assign_blocks(p, cache, pool, None, 0)
    model = Model(5, 9, 30, 7)
    model.step([0, 134, 135, 7 + 128 * 9, 500])
    same(cache, pool, model)
    K.kvarn_assign_blocks(p, cache, pool, None, 1)  # one of them would need a tenth block
    model.step([0, 134, 135, 7 + 128 * 9, 500], 1)
    assert model.err == 0
    same(cache, pool, model)
    K.kvarn_assign_blocks(p, cache, pool, None, 128)
    model.step([0, 134, 135, 7 + 128 * 9, 500], 128)
    assert model.err == 1
    same(cache, pool, model)


def test_whole_pool_handed_on(K):
    """A full pool whose holders end while others begin: every block changes hands within one call, in long rows."""
    p, cache, pool = make(K, 6, 700, 1500, 0)
    model = Model(6, 700, 1500, 0)
    for lengths in ([700 * 128, 0, 700 * 128, 0, 100 * 128, 0], [0, 650 * 128, 3 * 128, 699 * 128, 0, 148 * 128],
                    [128] * 6, [0] * 6, [250 * 128] * 6, [249 * 128, 255 * 128, 0, 0, 0, 600 * 128]):
        K.kvarn_assign_blocks(p, cache, pool, torch.tensor(lengths, dtype=torch.int32, device="cuda"), 0)
        model.step(lengths)
        assert model.err == 0
        same(cache, pool, model)


def test_pool_that_does_not_cover_the_growth(K):
    """From the first sequence on that does not fit, none grows; those that shrink and those that stay do."""
    p, cache, pool = make(K, 5, 20, 10, 0)
    model = Model(5, 20, 10, 0)
    for lengths in ([3 * 128, 0, 4 * 128, 0, 0], [4 * 128, 5 * 128, 3 * 128, 128, 128], [4 * 128, 3 * 128, 3 * 128, 0, 0]):
        K.kvarn_assign_blocks(p, cache, pool, torch.tensor(lengths, dtype=torch.int32, device="cuda"), 0)
        model.step(lengths)
        same(cache, pool, model)
    assert model.err == 1


def test_lengths_near_the_end_of_32_bits(K):
    p, cache, pool = make(K, 3, 4, 12, 0)
    model = Model(3, 4, 12, 0)
    lengths = [2**31 - 1, 512, 2**31 - 1]
    K.kvarn_assign_blocks(p, cache, pool, torch.tensor(lengths, dtype=torch.int32, device="cuda"), 2**31 - 1 - 512)
    model.step(lengths, 2**31 - 1 - 512)
    same(cache, pool, model)
    K.kvarn_assign_blocks(p, cache, pool, torch.tensor([-5, 513, -2**31], dtype=torch.int32, device="cuda"), 127)
    model.step([-5, 513, -2**31], 127)
    same(cache, pool, model)


def test_invalid_counts(K):
    """A count outside 0 .. max_blocks leaves its sequence, a ring that does not fit leaves all, unchanged (bit 3)."""
    p, cache, pool = make(K, 4, 8, 20, 0)
    n = torch.tensor([512] * 4, dtype=torch.int32, device="cuda")
    pool.n_blocks.copy_(torch.tensor([0, -1, 9, 0], dtype=torch.int32))
    K.kvarn_assign_blocks(p, cache, pool, n, 0)
    torch.cuda.synchronize()
    assert int(cache.err_word) == 8 and pool.n_blocks.tolist() == [4, -1, 9, 4] and pool.ring.tolist() == [8, 12, 0, 0]
    assert cache.block_table[1:3].unique().tolist() == [-1] and cache.block_table[3, :4].tolist() == [4, 5, 6, 7]
    for ring in ([20, 12], [-1, 12], [8, -1], [8, 21], [8, 20]):
        pool.n_blocks.copy_(torch.tensor([4, 0, 0, 4], dtype=torch.int32))
        pool.ring[:2] = torch.tensor(ring, dtype=torch.int32)
        cache.err_word.zero_()
        table, ids = cache.block_table.clone(), pool.free_ids.clone()
        K.kvarn_assign_blocks(p, cache, pool, torch.tensor([0, 128, 0, 0], dtype=torch.int32, device="cuda"), 0)
        torch.cuda.synchronize()
        assert int(cache.err_word) == 8 and pool.ring.tolist() == ring + [0, 0] and pool.n_blocks.tolist() == [4, 0, 0, 4]
        assert torch.equal(table, cache.block_table) and torch.equal(ids, pool.free_ids)


def test_rows_beyond_32_bits(K):
    """A table of 3 x 2^30 entries, the last sequences' rows behind 2^31 elements."""
    wide = 1 << 30
    p = K.kvarn_params_init(2)
    cache = K.Cache(p, 3, 1, 1, n_phys=4000)
    cache.max_blocks, cache.block_table = wide, torch.full((3, wide), -1, dtype=torch.int32, device="cuda")
    pool, model = K.BlockPool(cache), Model(3, 1300, 4000, 0)
    for lengths in ([5 * 128, 0, 1200 * 128], [0, 128, 1300 * 128], [700 * 128, 3 * 128, 0]):
        K.kvarn_assign_blocks(p, cache, pool, torch.tensor(lengths, dtype=torch.int32, device="cuda"), 0)
        model.step(lengths)
        torch.cuda.synchronize()
        for row, want in zip(cache.block_table, model.rows):
            assert row[:1301].tolist() == want + [-1] * (1301 - len(want))
        assert pool.n_blocks.tolist() == [len(r) for r in model.rows]
    cu = torch.tensor([0, 1, 2, 702 * 128 + 2], dtype=torch.int32, device="cuda")
    row = torch.empty(702 * 128 + 2, dtype=torch.int64, device="cuda")
    cache.block_table[2, :702] = torch.arange(702, dtype=torch.int32, device="cuda") + 7
    K.kvarn_token_map(p, cache, cu, None, row.numel(), None, None, row)
    torch.cuda.synchronize()
    at = torch.arange(702 * 128, device="cuda")
    assert torch.equal(row[2:], 3 * 128 + (at // 128 + 7) * 128 + at % 128)


def test_on_another_stream(K):
    p, cache, pool = make(K, 40, 12, 300, 0)
    model = Model(40, 12, 300, 0)
    other = torch.cuda.Stream()
    lengths = torch.arange(40, dtype=torch.int32, device="cuda") * 20
    cu = torch.cat([lengths.new_zeros(1), torch.cumsum(lengths, 0, dtype=torch.int32)])
    n = int(cu[-1])
    seq, pos, row = (torch.empty(n, dtype=dt, device="cuda") for dt in (torch.int32, torch.int32, torch.int64))
    torch.cuda.synchronize()
    K.kvarn_assign_blocks(p, cache, pool, lengths, 0, stream=other)
    K.kvarn_token_map(p, cache, cu, None, n, seq, pos, row, stream=other)
    other.synchronize()
    model.step(lengths.tolist())
    same(cache, pool, model)
    want = token_map(lengths.tolist(), [0] * 40, 0, 12, cache.block_table.cpu().numpy(), 300, n)
    for x, w in zip((seq, pos, row), want):
        assert np.array_equal(x.cpu().numpy(), w)


def test_replayed(K):
    """A captured call follows the lengths in its buffer, between eager ones."""
    p, cache, pool = make(K, 300, 12, 2000, 16)
    model = Model(300, 12, 2000, 16)
    n = torch.zeros(300, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        K.kvarn_assign_blocks(p, cache, pool, n, 1)
    rng = np.random.default_rng(3)
    for step in range(6):
        lengths = rng.integers(0, 900, 300)
        n.copy_(torch.from_numpy(lengths.astype(np.int32)))
        if step % 3 == 2:
            K.kvarn_assign_blocks(p, cache, pool, n, 1)
        else:
            g.replay()
        model.step(lengths, 1)
        same(cache, pool, model)


# ---- token maps --------------------------------------------------------------------------------


def token_map(counts, start, sink, max_blocks, table, n_phys, n_tokens):
    """seq, position, row of every token, -7 where nothing is written, and err_word."""
    batch, err = len(counts), 0
    seq, pos, row = np.full(n_tokens, -7), np.full(n_tokens, -7), np.full(n_tokens, -7, np.int64)
    t = 0
    for b, n in enumerate(counts):
        length = int(start[b]) + n
        for i in range(n):
            if t >= n_tokens:
                break
            at = int(start[b]) + i
            seq[t], pos[t], r = b, at if -2**31 <= at < 2**31 else -1, -1
            if 0 <= at < 2**31 - 1:
                blk = (at - sink) // 128
                if at < sink:
                    r = b * sink + at
                elif blk >= (length - sink) // 128:
                    r = batch * sink + b * 128 + (at - sink) % 128
                elif blk < max_blocks:
                    tile = b * max_blocks + blk if table is None else int(table[b, blk])
                    if table is not None and not 0 <= tile < n_phys:
                        err |= 2
                    else:
                        r = batch * (sink + 128) + tile * 128 + (at - sink) % 128
            row[t] = r
            t += 1
    return seq, pos, row, err


@pytest.mark.parametrize("paged", [True, False])
@pytest.mark.parametrize("sink", [0, 100])
@pytest.mark.parametrize("counts,more", [([1], 0), ([0, 0, 1, 0], 3), ([1023, 0, 2, 1024, 1], 0), ([300] * 70, 5), ([0] * 500 + [3000] + [0] * 500, 1),
                                         ([1, 0, 2, 5] * 1100, 0), ([0, 0], 4), ([7000], 0)])
def test_token_map(K, counts, more, sink, paged):
    rng = np.random.default_rng(len(counts))
    batch, total = len(counts), sum(counts)
    start = rng.integers(0, 700, batch).astype(np.int32)
    start[0] = 0
    max_blocks = 40
    p = K.kvarn_params_init(2, n_sink=sink)
    cache = K.Cache(p, batch, 1, 1, n_phys=9 if paged else 0)
    cache.max_blocks = max_blocks  # (only the table is looked at)
    table = rng.integers(-1, 10, (batch, max_blocks)).astype(np.int32) if paged else None
    cache.block_table = torch.from_numpy(table).cuda() if paged else None
    cu = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    n = total + more
    for use in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)):
        out = [torch.full((n + 1,), -7, dtype=dt, device="cuda") for dt in (torch.int32, torch.int32, torch.int64)]
        cache.err_word.zero_()
        K.kvarn_token_map(p, cache, cu, torch.from_numpy(start).cuda(), n, *[x if u else None for x, u in zip(out, use)])
        torch.cuda.synchronize()
        *want, err = token_map(counts, start, sink, max_blocks, table, 9, n)
        for x, w, u in zip(out, want, use):
            assert int(x[n]) == -7 and np.array_equal(x[:n].cpu().numpy(), w if u else np.full(n, -7))
        assert int(cache.err_word) == (err if use[2] else 0)


def test_token_map_of_part_of_the_rows_and_far_positions(K):
    p = K.kvarn_params_init(2)
    cache = K.Cache(p, 3, 1, 1, n_phys=1)
    cache.max_blocks, cache.n_phys = 3, 1
    cache.block_table = torch.zeros((3, 3), dtype=torch.int32, device="cuda")
    start = np.array([2**31 - 3, -4, 0], np.int32)
    counts = [5, 9, 6]
    cu = torch.tensor([0, 5, 14, 20], dtype=torch.int32, device="cuda")
    for n in (20, 17, 3):  # (outputs that hold fewer rows than there are tokens)
        out = [torch.full((21,), -7, dtype=dt, device="cuda") for dt in (torch.int32, torch.int32, torch.int64)]
        K.kvarn_token_map(p, cache, cu, torch.from_numpy(start).cuda(), n, *out)
        torch.cuda.synchronize()
        *want, _ = token_map(counts, start, 0, 3, cache.block_table.cpu().numpy(), 1, n)
        for x, w in zip(out, want):
            assert np.array_equal(x[:n].cpu().numpy(), w) and bool((x[n:] == -7).all())
    out = [torch.full((21,), -7, dtype=torch.int32, device="cuda") for _ in range(2)]
    K.kvarn_token_map(p, cache, cu, None, 20, *out, None)
    torch.cuda.synchronize()
    assert out[1][:20].tolist() == [0, 1, 2, 3, 4, 0, 1, 2, 3, 4, 5, 6, 7, 8, 0, 1, 2, 3, 4, 5]
