"""Block tables and slot maps (tt_blocks_extend, tt_blocks_release) against a plain restatement: whole numbers, every entry equal,
and everything that the calls may not write as it was."""
import numpy as np
import pytest


@pytest.fixture(scope="module")
def tt():
    from paper_2607_29678_b200 import build
    build.build()
    import paper_2607_29678_b200 as m
    return m


# ---- a plain restatement, request by request ----------------------------------------------------------------------


class Pool:
    """Lists in place of device memory."""

    def __init__(self, table, seq_len, free, n_free, block):
        self.table, self.seq, self.free, self.n_free, self.block = table.copy(), seq_len.astype(np.int64).copy(), free.copy(), int(n_free), block

    def blocks(self, tokens):
        return -(-tokens // self.block)

    def extend(self, new_off):
        """(slots, positions, requests)"""
        slots, pos, req = [], [], []
        for r in range(self.seq.size):
            n = int(new_off[r + 1] - new_off[r])
            for b in range(int(self.blocks(self.seq[r])), int(self.blocks(self.seq[r] + n))):
                self.n_free -= 1
                self.table[r, b] = self.free[self.n_free]
            p = np.arange(self.seq[r], self.seq[r] + n)
            slots.append(self.table[r, p // self.block].astype(np.int64) * self.block + p % self.block if n else np.zeros(0, np.int64))
            pos.append(p)
            req.append(np.full(n, r))
            self.seq[r] += n
        cat = lambda v: np.concatenate(v) if v else np.zeros(0, np.int64)  # noqa: E731
        return cat(slots), cat(pos), cat(req)

    def release(self, keep):
        gone = []
        for r in range(self.seq.size):
            gone += list(self.table[r, int(self.blocks(keep[r])):int(self.blocks(self.seq[r]))])
            self.seq[r] = keep[r]
        for b in reversed(gone):
            self.free[self.n_free] = b
            self.n_free += 1


def test_restatement_by_hand():
    p = Pool(np.full((2, 4), -1, np.int32), np.array([0, 0]), np.arange(10, 16, dtype=np.int32), 6, 4)
    slots, pos, req = p.extend([0, 5, 6])
    assert list(p.table[0]) == [15, 14, -1, -1] and list(p.table[1]) == [13, -1, -1, -1] and p.n_free == 3
    assert list(slots) == [60, 61, 62, 63, 56, 52] and list(pos) == [0, 1, 2, 3, 4, 0] and list(req) == [0] * 5 + [1]
    slots, _, _ = p.extend([0, 1, 4])
    assert list(slots) == [57, 53, 54, 55] and p.n_free == 3
    p.release(np.array([4, 0]))
    assert p.n_free == 5 and list(p.free[:5]) == [10, 11, 12, 13, 14]


def test_refusals_without_a_device(tt):
    L, a = tt.lib(), 0x1000

    def ext(off=a, n=3, seq=a, block=16, table=a, width=4, free=a, cap=8, nf=a, slots=a, scap=8, seq_out=a, nf_out=a, status=a, ws=a, ws_bytes=1 << 20):
        return L.tt_blocks_extend(off, n, seq, block, table, width, free, cap, nf, None, slots, scap, None, None, seq_out, nf_out, status, ws, ws_bytes)

    def rel(keep=a, n=3, seq=a, block=16, table=a, width=4, free=a, cap=8, nf=a, seq_out=a, nf_out=a, status=a, ws=a, ws_bytes=1 << 20):
        return L.tt_blocks_release(keep, n, seq, block, table, width, free, cap, nf, None, seq_out, nf_out, status, ws, ws_bytes)

    both = [dict(n=1 << 24, ws_bytes=1 << 40), dict(seq=None), dict(block=0), dict(block=1 << 31), dict(table=None), dict(width=1 << 31), dict(free=None), dict(cap=1 << 31), dict(nf=None),
            dict(seq_out=None), dict(nf_out=None), dict(status=None), dict(ws=None), dict(ws=a + 16), dict(ws_bytes=tt.lib().tt_blocks_workspace_bytes(3) - 1)]
    both += [dict(seq=a + 2), dict(table=a + 1), dict(free=a + 2), dict(nf=a + 4), dict(seq_out=a + 2), dict(nf_out=a + 4), dict(status=a + 2)]
    for kw in both + [dict(off=None), dict(off=a + 4), dict(slots=None), dict(slots=a + 4), dict(scap=1 << 31)]:
        assert ext(**kw) == tt.TT_ERR_ARG, kw
    for kw in both + [dict(keep=None), dict(keep=a + 2)]:
        assert rel(**kw) == tt.TT_ERR_ARG, kw
    import torch
    with pytest.raises(ValueError):
        tt.blocks_extend(torch.zeros(3, dtype=torch.int64), *[dict(tt.alloc_blocks(2, 4, 8, 8, device="cpu")[0])], 16, tt.alloc_blocks(2, 4, 8, 8, device="cpu")[1])


# ---- on the GPU ----------------------------------------------------------------------------------------------------


def cuda(a, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def setup(n, block, old, extra_blocks, width, seed, n_used_only=False):
    """(Pool, state on the device): requests with `old` tokens, a shuffled free list with `extra_blocks` blocks left."""
    import torch
    rng = np.random.default_rng(seed)
    have = -(-old // block)
    used = int(have.sum())
    total = used + extra_blocks
    ids = rng.permutation(total).astype(np.int32)
    table = np.full((n, width), -1, np.int32)
    table[np.arange(width)[None, :] < have[:, None]] = ids[:used]
    free = np.full(total, -9, np.int32)
    free[:extra_blocks] = ids[used:]
    pool = Pool(table, old, free, extra_blocks, block)
    state = dict(block_table=cuda(table, torch.int32), seq_len=cuda(old, torch.int32), free_blocks=cuda(free, torch.int32), n_free=cuda(np.array([extra_blocks]), torch.int64))
    return pool, state


def buffers(tt, state, cap, in_place):
    import torch
    n = state["seq_len"].numel()
    i = dict(dtype=torch.int32, device="cuda")
    return dict(slots=torch.full((cap,), -5, dtype=torch.int64, device="cuda"), positions=torch.full((cap,), -5, **i), requests=torch.full((cap,), -5, **i),
                seq_len=state["seq_len"] if in_place else torch.full((n,), -5, **i), n_free=state["n_free"] if in_place else torch.full((1,), -5, dtype=torch.int64, device="cuda"),
                status=torch.full((1,), -5, **i), workspace=torch.full((int(tt.lib().tt_blocks_workspace_bytes(n)),), 0xEE, dtype=torch.uint8, device="cuda"))


def agree(pool, state, bufs, maps=None, status=0):
    import torch
    torch.cuda.synchronize()
    assert int(bufs["status"].item()) == status
    assert np.array_equal(state["block_table"].cpu().numpy(), pool.table)
    assert np.array_equal(state["free_blocks"].cpu().numpy(), pool.free)
    assert np.array_equal(bufs["seq_len"].cpu().numpy(), pool.seq) and int(bufs["n_free"].item()) == pool.n_free
    if maps is not None:
        n = maps[0].size
        for name, want in zip(("slots", "positions", "requests"), maps):
            got = bufs[name].cpu().numpy()
            assert np.array_equal(got[:n], want), name
            assert (got[n:] == -5).all(), name


CASES = [  # requests, block, most new tokens, most old tokens, seed
    (1, 16, 1, 0, 0), (1, 1, 5, 3, 1), (2, 16, 40, 33, 2), (7, 3, 20, 9, 3), (33, 16, 1, 500, 4), (256, 16, 1, 4_000, 5), (1_000, 16, 300, 900, 6), (1_025, 64, 30, 10, 7), (5, 128, 9_000, 1_000, 8),
    (1, 16, 70_000, 5, 9), (3, 48, 100_000, 0, 10), (3_000, 7, 90, 60, 11), (64, 1, 2_000, 100, 12), (20_000, 16, 3, 40, 13), (2, 1 << 20, 3_000, 3_000, 14), (40_000, 5, 25, 9, 15)]


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,block,most_new,most_old,seed", CASES)
def test_extend_and_release(tt, n, block, most_new, most_old, seed, in_place):
    import torch
    rng = np.random.default_rng(seed)
    old = rng.integers(0, most_old + 1, n)
    new = rng.integers(0, most_new + 1, n)
    if n > 4:
        new[rng.integers(0, n, n // 4)] = 0
        new[0] = new[-1] = 0
    if new.sum() == 0:
        new[-1] = 1
    off = np.r_[0, np.cumsum(new)]
    need = int((-(-(old + new) // block) - (-(-old // block))).sum())
    width = int((-(-(old + new) // block)).max()) + 1
    pool, state = setup(n, block, old, need + (seed % 3), width, seed)     # (every third case takes the last block)
    bufs = buffers(tt, state, int(off[-1]) + 37, in_place)
    first = pool.free.copy(), pool.n_free
    maps = pool.extend(off)
    tt.blocks_extend(cuda(off, torch.int64), state, block, bufs)
    agree(pool, state, bufs, maps)
    # part of every request goes back, then all of it
    now = dict(state, seq_len=bufs["seq_len"], n_free=bufs["n_free"])
    keep = rng.integers(0, pool.seq + 1)
    out = buffers(tt, now, 1, in_place)
    pool.release(keep)
    tt.blocks_release(cuda(keep, torch.int32), now, block, out)
    agree(pool, now, out)
    now = dict(now, seq_len=out["seq_len"], n_free=out["n_free"])
    out = buffers(tt, now, 1, in_place)
    pool.release(np.zeros(n, np.int64))
    tt.blocks_release(torch.zeros(n, dtype=torch.int32, device="cuda"), now, block, out)
    agree(pool, now, out)
    assert pool.n_free == pool.free.size and first[1] <= pool.n_free
    assert sorted(pool.free) == list(range(pool.free.size))


@pytest.mark.gpu
def test_release_undoes_extend(tt):
    import torch
    rng = np.random.default_rng(3)
    old, new = rng.integers(0, 100, 50), rng.integers(0, 100, 50)
    pool, state = setup(50, 16, old, 1_000, 40, 3)
    bufs = buffers(tt, state, int(new.sum()), True)
    free = state["free_blocks"].clone()
    tt.blocks_extend(cuda(np.r_[0, np.cumsum(new)], torch.int64), state, 16, bufs)
    assert int(state["n_free"].item()) < 1_000
    tt.blocks_release(cuda(old, torch.int32), state, 16, bufs)
    assert int(state["n_free"].item()) == 1_000 and torch.equal(state["free_blocks"], free) and np.array_equal(state["seq_len"].cpu().numpy(), old)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [5, 1_300, 20_000])
@pytest.mark.parametrize("in_place", [False, True])
def test_a_refused_call_changes_nothing(tt, n, in_place):
    import torch
    rng = np.random.default_rng(n)
    old, new = rng.integers(0, 50, n), rng.integers(1, 50, n)
    off = np.r_[0, np.cumsum(new)]
    need = int((-(-(old + new) // 16) - (-(-old // 16))).sum())
    mid = n // 2

    def refused(status, off=off, old=old, spare=0, width=8, cap=None, n_free=None):
        pool, state = setup(n, 16, np.clip(old, 0, 120), need + spare, width, 1)
        state["seq_len"].copy_(cuda(old, torch.int32)); pool.seq = old.copy()
        if n_free is not None:
            state["n_free"].fill_(n_free); pool.n_free = n_free
        bufs = buffers(tt, state, int(np.max(off)) if cap is None else cap, in_place)
        tt.blocks_extend(cuda(off, torch.int64), state, 16, bufs)
        agree(pool, state, bufs, (np.zeros(0), np.zeros(0), np.zeros(0)), status)

    def changed(v, at, to):
        v = v.copy(); v[at] = to
        return v

    refused(tt.TT_ERR_CAPACITY, spare=-1)
    refused(tt.TT_ERR_CAPACITY, cap=int(off[-1]) - 1)
    refused(tt.TT_ERR_CAPACITY, old=changed(old, mid, 16 * 8 - int(new[mid]) + 1))
    refused(tt.TT_ERR_CAPACITY, old=changed(old, mid, 2**31 - 1))
    refused(tt.TT_ERR_ARG, off=off + 1, spare=5)
    refused(tt.TT_ERR_ARG, off=changed(off, mid, -1))
    refused(tt.TT_ERR_ARG, off=changed(off, mid, int(off[mid + 1]) + 1), spare=5)
    refused(tt.TT_ERR_ARG, old=changed(old, mid, -1))
    refused(tt.TT_ERR_ARG, n_free=-1)
    refused(tt.TT_ERR_ARG, n_free=2**40)
    refused(tt.TT_ERR_ARG, old=changed(old, mid, -1), spare=-1)             # an argument comes before the capacity

    def kept(status, keep, old=old, room=0, n_free=None):
        pool, state = setup(n, 16, np.clip(old, 0, 120), 7, 8, 1)
        state["seq_len"].copy_(cuda(old, torch.int32)); pool.seq = old.copy()
        if room:
            state["free_blocks"] = state["free_blocks"][:room].clone(); pool.free = pool.free[:room]
        if n_free is not None:
            state["n_free"].fill_(n_free); pool.n_free = n_free
        bufs = buffers(tt, state, 1, in_place)
        tt.blocks_release(cuda(keep, torch.int32), state, 16, bufs)
        agree(pool, state, bufs, None, status)

    kept(tt.TT_ERR_ARG, changed(old, mid, int(old[mid]) + 1))
    kept(tt.TT_ERR_ARG, changed(old, mid, -1))
    kept(tt.TT_ERR_ARG, np.zeros(n, np.int64), old=changed(old, mid, -3))
    kept(tt.TT_ERR_CAPACITY, np.zeros(n, np.int64), old=changed(old, mid, 16 * 8 + 1))
    kept(tt.TT_ERR_CAPACITY, np.zeros(n, np.int64), room=7)
    kept(tt.TT_ERR_ARG, np.zeros(n, np.int64), n_free=10**12)


@pytest.mark.gpu
def test_no_requests_and_no_tokens(tt):
    import torch
    for n in (0, 3):
        pool, state = setup(n, 16, np.full(n, 5), 4, 2, 1)
        bufs = buffers(tt, state, 4, False)
        tt.blocks_extend(torch.zeros(n + 1, dtype=torch.int64, device="cuda"), state, 16, bufs)
        agree(pool, state, bufs, (np.zeros(0), np.zeros(0), np.zeros(0)))
        bufs = buffers(tt, state, 4, False)
        tt.blocks_release(state["seq_len"].clone(), state, 16, bufs)
        agree(pool, state, bufs)
    # maps that are not wanted, a map without room
    pool, state = setup(3, 16, np.full(3, 5), 4, 2, 1)
    bufs = buffers(tt, state, 40, False)
    maps = pool.extend([0, 20, 20, 21])
    off = cuda(np.array([0, 20, 20, 21]), torch.int64)
    tt.blocks_extend(off, state, 16, {k: v for k, v in bufs.items() if k not in ("positions", "requests")})
    torch.cuda.synchronize()
    assert np.array_equal(bufs["slots"].cpu().numpy()[:21], maps[0]) and (bufs["positions"] == -5).all()
    pool, state = setup(2, 16, np.full(2, 5), 4, 2, 1)
    bufs = buffers(tt, state, 0, False)
    tt.blocks_extend(torch.zeros(3, dtype=torch.int64, device="cuda"), state, 16, bufs)
    agree(pool, state, bufs, (np.zeros(0), np.zeros(0), np.zeros(0)))


@pytest.mark.gpu
def test_slots_beyond_32_bits_and_long_requests(tt):
    """Block ids near 2^31 (they are not looked at), requests of up to 2^31 - 1 tokens."""
    import torch
    block, big = 1 << 16, 2**31 - 1
    state = dict(block_table=torch.full((2, 32_768), 2**31 - 5, dtype=torch.int32, device="cuda"), seq_len=cuda(np.array([big - 3, 0]), torch.int32),
                 free_blocks=cuda(np.array([2**31 - 1, 2**31 - 2]), torch.int32), n_free=cuda(np.array([2]), torch.int64))
    bufs = buffers(tt, state, 8, False)
    tt.blocks_extend(cuda(np.array([0, 3, 5]), torch.int64), state, block, bufs)
    torch.cuda.synchronize()
    assert int(bufs["status"].item()) == 0 and bufs["seq_len"].tolist() == [big, 2] and int(bufs["n_free"].item()) == 1
    want = [(2**31 - 5) * block + (big - 3 + i) % block for i in range(3)] + [(2**31 - 2) * block + i for i in range(2)]
    assert bufs["slots"].tolist()[:5] == want and bufs["positions"].tolist()[:3] == [big - 3, big - 2, big - 1]
    tt.blocks_extend(cuda(np.array([0, 4, 5]), torch.int64), state, block, bufs)
    torch.cuda.synchronize()
    assert int(bufs["status"].item()) == tt.TT_ERR_CAPACITY


@pytest.mark.gpu
def test_decode_steps_replayed_from_a_graph(tt):
    """One captured step in place, replayed: every replay moves the conversations on; two graphs share the workspace in turn."""
    import torch
    n = 37
    old = np.random.default_rng(1).integers(0, 60, n)
    pool, state = setup(n, 16, old, 400, 12, 1)
    one = torch.arange(n + 1, dtype=torch.int64, device="cuda")
    bufs = buffers(tt, state, n, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tt.blocks_extend(one, state, 16, bufs)
    side.synchronize()
    agree(pool, state, bufs, pool.extend(np.arange(n + 1)))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            tt.blocks_extend(one, state, 16, bufs)
        graphs.append(g)
    for step in range(40):
        graphs[step % 2].replay()
        agree(pool, state, bufs, pool.extend(np.arange(n + 1)))


@pytest.mark.gpu
@pytest.mark.parametrize("n,share", [(30_000, 0.02), (9_000, 0.3), (2_500, 0.001), (100_000, 0.0005)])
def test_most_requests_get_nothing(tt, n, share):
    """Thousands of requests without a new token between those with some, and of requests that give no block back."""
    import torch
    rng = np.random.default_rng(n)
    old = rng.integers(0, 40, n)
    new = np.where(rng.random(n) < share, rng.integers(1, 120, n), 0)
    new[n // 2] = 3_000
    off = np.r_[0, np.cumsum(new)]
    need = int((-(-(old + new) // 16) - (-(-old // 16))).sum())
    pool, state = setup(n, 16, old, need, 200, n)
    bufs = buffers(tt, state, int(off[-1]), True)
    maps = pool.extend(off)
    tt.blocks_extend(cuda(off, torch.int64), state, 16, bufs)
    agree(pool, state, bufs, maps)
    keep = np.where(rng.random(n) < 0.9, pool.seq, pool.seq // 2)
    pool.release(keep)
    tt.blocks_release(cuda(keep, torch.int32), state, 16, bufs)
    agree(pool, state, bufs)


@pytest.mark.gpu
@pytest.mark.parametrize("n,most", [(40, 30), (5, 60_000), (3_000, 90)])
def test_maps_at_odd_addresses(tt, n, most):
    import torch
    rng = np.random.default_rng(n)
    old, new = rng.integers(0, 50, n), rng.integers(0, most, n)
    off = np.r_[0, np.cumsum(new)]
    need = int((-(-(old + new) // 16) - (-(-old // 16))).sum())
    width = int((-(-(old + new) // 16)).max()) + 1
    total = int(off[-1])
    for shift in (1, 2, 3):
        pool, state = setup(n, 16, old, need, width, n)
        whole = {"slots": torch.full((total + 8,), -5, dtype=torch.int64, device="cuda"), "positions": torch.full((total + 8,), -5, dtype=torch.int32, device="cuda"),
                 "requests": torch.full((total + 8,), -5, dtype=torch.int32, device="cuda")}
        bufs = dict(buffers(tt, state, total, False), **{k: v[shift:shift + total] for k, v in whole.items()})
        maps = pool.extend(off)
        tt.blocks_extend(cuda(off, torch.int64), state, 16, bufs)
        agree(pool, state, bufs, maps)
        for v in whole.values():
            assert (v[:shift] == -5).all() and (v[shift + total:] == -5).all()


@pytest.mark.gpu
def test_two_pools_on_two_streams(tt):
    """Calls on different pools and workspaces do not meet; large ones captured, with both directions in one graph."""
    import torch
    pools, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(2):
        rng = np.random.default_rng(k)
        n = 3_000 + k
        old, new = rng.integers(0, 60, n), rng.integers(0, 90, n)
        off = np.r_[0, np.cumsum(new)]
        pool, state = setup(n, 16, old, 40_000, 16, k)
        pools.append((pool, state, buffers(tt, state, int(off[-1]), True), off, cuda(off, torch.int64), cuda(old, torch.int32), old))
    torch.cuda.synchronize()
    for _ in range(3):
        for st, (pool, state, bufs, off, d_off, d_old, old) in zip(streams, pools):
            with torch.cuda.stream(st):
                tt.blocks_extend(d_off, state, 16, bufs)
                tt.blocks_release(d_old, state, 16, bufs)
    torch.cuda.synchronize()
    for pool, state, bufs, off, d_off, d_old, old in pools:
        maps = pool.extend(off)
        pool.release(old)
        agree(pool, state, bufs, maps)
    pool, state, bufs, off, d_off, d_old, old = pools[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        tt.blocks_extend(d_off, state, 16, bufs)
        tt.blocks_release(d_old, state, 16, bufs)
        tt.blocks_extend(d_off, state, 16, bufs)
        tt.blocks_release(d_old, state, 16, bufs)
    bufs["slots"].fill_(-5)
    graph.replay()
    torch.cuda.synchronize()
    want = Pool(pool.table, pool.seq, pool.free, pool.n_free, 16)
    slots, _, _ = want.extend(off)
    assert np.array_equal(bufs["slots"].cpu().numpy(), slots) and np.array_equal(state["seq_len"].cpu().numpy(), old) and int(state["n_free"].item()) == pool.n_free
