"""hma_step_tables, hma_release_pages, hma_rope_table: against a sequence-by-sequence statement of the same rules."""
import numpy as np
import pytest
import torch

from paper_2606_29986_b200 import hma


def step_oracle(past, new, table, free, count, max_tokens, num_pages):
    """Everything hma_step_tables writes, and the flag it raises (0: none), one token at a time."""
    past, new, table = [int(x) for x in past], [int(x) for x in new], table.copy()
    B, max_pages = table.shape
    refused = dict(table=table, context=np.array(past, np.int64), starts=np.zeros(B + 1, np.int64), positions=np.zeros(max_tokens, np.int64),
                   slots=np.full(max_tokens, -1, np.int64), left=count)
    if any(p < 0 or n < 0 or p + n > max_pages * 16 for p, n in zip(past, new)) or sum(new) > max_tokens:
        return refused, hma.HMA_FLAG_BAD_LENGTHS
    need = sum((p + n + 15) // 16 - (p + 15) // 16 for p, n in zip(past, new))
    if count < 0 or count > num_pages or need > count:
        return refused, hma.HMA_FLAG_NO_PAGES
    got = dict(table=table, context=np.array([p + n for p, n in zip(past, new)], np.int64), starts=np.zeros(B + 1, np.int64),
               positions=np.zeros(max_tokens, np.int64), slots=np.full(max_tokens, -1, np.int64), left=count - need)
    top, i = count, 0
    for b, (p, n) in enumerate(zip(past, new)):
        for page in range((p + 15) // 16, (p + n + 15) // 16):
            top -= 1
            table[b, page] = free[top]
        for t in range(p, p + n):
            got["positions"][i] = t
            page = int(table[b, t // 16])
            got["slots"][i] = page * 16 + t % 16 if page >= 0 else -2
            i += 1
        got["starts"][b + 1] = i
    return got, 0


class Pool:
    """A page pool with `held` tokens per sequence already placed, as numpy and on the GPU."""

    def __init__(self, past, max_pages, spare, seed=0):
        rng = np.random.default_rng(seed)
        pages = [(max(int(p), 0) + 15) // 16 for p in past]
        self.num_pages = sum(pages) + spare
        ids = rng.permutation(self.num_pages).astype(np.int32)
        self.table = np.full((len(past), max_pages), -1, np.int32)
        o = 0
        for b, n in enumerate(pages):
            n = min(n, max_pages)
            self.table[b, :n] = ids[o:o + n]
            o += n
        self.count = self.num_pages - o
        self.free = np.concatenate([ids[o:], np.full(o, -7, np.int32)])
        self.past = np.array(past, np.int32)

    def gpu(self):
        self.cache = hma.KVCache(hma.make_desc(1, 8, 8, self.num_pages))
        return [torch.from_numpy(x.copy()).cuda() for x in (self.past, self.table, self.free, np.array([self.count], np.int32))]


def run_step(pool, new, max_tokens, in_place=False):
    past, table, free, count = pool.gpu()
    B = len(pool.past)
    guard = 3
    ctx = past if in_place else torch.full((B,), -9, dtype=torch.int32, device="cuda")
    left = count if in_place else torch.full((1,), -9, dtype=torch.int32, device="cuda")
    starts = torch.full((B + 1 + guard,), -9, dtype=torch.int32, device="cuda")
    pos = torch.full((max_tokens + guard,), -9, dtype=torch.int32, device="cuda")
    slots = torch.full((max_tokens + guard,), -9, dtype=torch.int64, device="cuda")
    hma.hma_step_tables(pool.cache, past, torch.tensor(new, dtype=torch.int32, device="cuda"), table, free, count, ctx,
                        starts[:B + 1], pos[:max_tokens], slots[:max_tokens], left)
    torch.cuda.synchronize()
    for t in (starts[B + 1:], pos[max_tokens:], slots[max_tokens:]):
        assert bool((t == -9).all())
    assert np.array_equal(free.cpu().numpy(), pool.free)
    if not in_place:
        assert np.array_equal(past.cpu().numpy(), pool.past) and int(count) == pool.count
    return dict(table=table.cpu().numpy(), context=ctx.cpu().numpy(), starts=starts[:B + 1].cpu().numpy(), positions=pos[:max_tokens].cpu().numpy(),
                slots=slots[:max_tokens].cpu().numpy(), left=int(left))


def check_step(pool, new, max_tokens, flag=0, in_place=False):
    want, want_flag = step_oracle(pool.past, new, pool.table, pool.free, pool.count, max_tokens, pool.num_pages)
    assert want_flag == flag
    got = run_step(pool, new, max_tokens, in_place)
    for k in want:
        assert np.array_equal(got[k], want[k]), k
    assert hma.hma_error_flags(pool.cache) == flag


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("past,new,pad", [
    ([0], [1], 0), ([15], [1], 1), ([16], [1], 0), ([0], [0], 4), ([7, 0, 31, 16], [1, 33, 1, 0], 5),
    ([100, 5, 0, 0, 64], [0, 0, 0, 1, 16], 2), ([3] * 33, [1] * 33, 0)])
def test_step_small(past, new, pad, in_place):
    check_step(Pool(past, 40, 20), new, sum(new) + pad, in_place=in_place)


@pytest.mark.gpu
@pytest.mark.parametrize("batch,most,pad", [(1024, 3, 17), (1000, 1, 0), (257, 90, 1000), (5, 4000, 3), (1, 16000, 0), (32, 129, 4097)])
def test_step_random(batch, most, pad):
    rng = np.random.default_rng(batch)
    past = rng.integers(0, 900, batch)
    new = rng.integers(0, most + 1, batch).astype(np.int32)
    new[-1] = most
    pool = Pool(past, 60 + most // 16 + 2, int((new // 16 + 2).sum()), seed=batch)
    check_step(pool, new, int(new.sum()) + pad)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("past,new,max_tokens,max_pages,spare,flag", [
    ([5, 16], [1, 1], 2, 8, 0, 128), ([5, 16], [1, 17], 18, 8, 1, 128), ([-1, 4], [1, 1], 2, 8, 4, 256), ([1, 4], [1, -1], 2, 8, 4, 256),
    ([1, 120], [1, 9], 16, 8, 9, 256), ([1, 2], [3, 3], 5, 8, 9, 256), ([2**31 - 1], [2**31 - 1], 5, 8, 9, 256), ([4, 9], [1, 8191], 8192, 600, 100, 128)])
def test_step_is_refused_as_a_whole(past, new, max_tokens, max_pages, spare, flag, in_place):
    pool = Pool([min(p, 128) for p in past], max_pages, spare)
    pool.past = np.array(past, np.int32)
    check_step(pool, new, max_tokens, flag=flag, in_place=in_place)


@pytest.mark.gpu
def test_step_exactly_uses_the_pool_and_the_table():
    check_step(Pool([0, 17], 8, 13), [128, 111], 300, flag=hma.HMA_FLAG_NO_PAGES)       # 8 + 6 pages needed
    check_step(Pool([0, 17], 8, 14), [128, 111], 300)                                   # the last page, and the last token of the table


@pytest.mark.gpu
def test_bad_free_counts_and_missing_pages():
    for count in (-1, 10**6):
        pool = Pool([5], 8, 4)
        pool.count = count
        check_step(pool, [40], 40, flag=hma.HMA_FLAG_NO_PAGES)
    pool = Pool([5, 20], 8, 4)
    pool.table[1, 1] = -1                                                      # the page that the next token belongs in is missing
    check_step(pool, [1, 1], 2)


@pytest.mark.gpu
def test_steps_and_releases_together():
    """Some hundred steps of a small serving loop on the GPU; no page is ever held twice, and all come back."""
    rng = np.random.default_rng(3)
    B, max_pages, N = 6, 12, 40
    cache = hma.KVCache(hma.make_desc(1, 8, 8, N))
    i32 = dict(dtype=torch.int32, device="cuda")
    table, ctx = torch.full((B, max_pages), -1, **i32), torch.zeros(B, **i32)
    free, count = torch.randperm(N, device="cuda").int(), torch.tensor([N], **i32)
    starts, pos, slots = torch.zeros(B + 1, **i32), torch.zeros(64, **i32), torch.zeros(64, dtype=torch.int64, device="cuda")
    lens = np.zeros(B, np.int64)
    for _ in range(150):
        new = rng.integers(0, 9, B) * (lens < 150)
        new_t = torch.tensor(new, **i32)
        before = table.cpu().numpy().copy()
        hma.hma_step_tables(cache, ctx, new_t, table, free, count, ctx, starts, pos, slots)
        flags = hma.hma_error_flags(cache)
        if flags:
            assert flags == hma.HMA_FLAG_NO_PAGES and np.array_equal(before, table.cpu().numpy()) and bool((slots == -1).all())
        else:
            lens += new
        assert np.array_equal(ctx.cpu().numpy(), lens)
        done = (rng.random(B) < (0.5 if flags else 0.05)).astype(np.int32)
        if done.any():
            hma.hma_release_pages(cache, torch.tensor(done, **i32), ctx, table, free, count)
            lens[done != 0] = 0
        t = table.cpu().numpy()
        used = [int(t[b, p]) for b in range(B) for p in range((int(lens[b]) + 15) // 16)]
        rest = free[:int(count)].cpu().numpy().tolist()
        assert sorted(used + rest) == list(range(N))
        assert (np.sort(t, axis=1)[:, ::-1][:, 0] < N).all() and np.array_equal(ctx.cpu().numpy(), lens)
    assert hma.hma_error_flags(cache) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("past,most", [([40, 7, 100], 9), ([33000, 5, 16384, 0, 700], 2100)])
def test_release_passes_over_entries_that_name_no_page(past, most):
    """Pages given up behind a window: their entries (-1, or anything outside the cache) do not reach the free list."""
    pool, rng = Pool(past, most, 5, seed=1), np.random.default_rng(2)
    gone = [1] * (len(past) - 1) + [0]
    for b, n in enumerate(past):
        k = np.flatnonzero(rng.random((n + 15) // 16) < 0.4)
        pool.table[b, k] = rng.choice([-1, -5, pool.num_pages, 2**31 - 1], len(k))
    named = [[int(x) for x in pool.table[b, :(n + 15) // 16] if 0 <= x < pool.num_pages] for b, n in enumerate(past)]
    back = [x for b in range(len(past)) if gone[b] for x in named[b]]
    for n in (0, pool.count, pool.num_pages - len(back), pool.num_pages - len(back) + 1):      # at most num_pages fit: the last one is refused
        ctx, table, free, count = pool.gpu()
        count.fill_(n)
        hma.hma_release_pages(pool.cache, torch.tensor(gone, dtype=torch.int32, device="cuda"), ctx, table, free, count)
        want_table, want_free, want_ctx, want_n = pool.table.copy(), pool.free.copy(), np.array(past), n
        if n + len(back) <= pool.num_pages:
            for b, t in enumerate(past):
                if gone[b]:
                    want_table[b, :(t + 15) // 16] = -1
                    want_ctx[b] = 0
            want_free[n:n + len(back)] = back
            want_n = n + len(back)
        assert int(count) == want_n and np.array_equal(ctx.cpu().numpy(), want_ctx)
        assert np.array_equal(table.cpu().numpy(), want_table) and np.array_equal(free.cpu().numpy(), want_free)
        assert hma.hma_error_flags(pool.cache) == (0 if n + len(back) <= pool.num_pages else 128)


@pytest.mark.gpu
def test_release_refusals_change_nothing():
    pool = Pool([40, 7], 4, 3)
    past, table, free, count = pool.gpu()
    one = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    for ctx, n, flag in (([65, 7], pool.count, 256), ([-1, 7], pool.count, 256), ([40, 7], pool.num_pages - 2, 128), ([40, 7], -1, 128)):
        c = torch.tensor(ctx, dtype=torch.int32, device="cuda")
        count.fill_(n)
        hma.hma_release_pages(pool.cache, one, c, table, free, count)
        assert hma.hma_error_flags(pool.cache) == flag and int(count) == n and c.tolist() == ctx
        assert np.array_equal(table.cpu().numpy(), pool.table) and np.array_equal(free.cpu().numpy(), pool.free)
    count.fill_(pool.count)
    c = torch.tensor([40, -1], dtype=torch.int32, device="cuda")               # an unfinished sequence is not looked at
    hma.hma_release_pages(pool.cache, one, c, table, free, count)
    assert int(count) == pool.count + 3 and c.tolist() == [0, -1] and hma.hma_error_flags(pool.cache) == 0
    assert np.array_equal(free[pool.count:pool.count + 3].cpu().numpy(), pool.table[0, :3])


@pytest.mark.gpu
def test_step_in_a_graph_and_on_another_stream():
    pool = Pool([15, 0, 40], 600, 2000)
    past, table, free, count = pool.gpu()
    i32 = dict(dtype=torch.int32, device="cuda")
    new, starts = torch.zeros(3, **i32), torch.zeros(4, **i32)
    pos, slots = torch.zeros(9000, **i32), torch.zeros(9000, dtype=torch.int64, device="cuda")
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        hma.hma_step_tables(pool.cache, past, new, table, free, count, past, starts, pos, slots)
    lens = pool.past.astype(np.int64)
    for step in ([1, 1, 1], [1, 8000, 0], [3, 2, 1]):
        want, flag = step_oracle(lens, step, table.cpu().numpy(), pool.free, int(count), 9000, pool.num_pages)
        assert flag == 0
        new.copy_(torch.tensor(step, **i32))
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(table.cpu().numpy(), want["table"]) and np.array_equal(slots.cpu().numpy(), want["slots"])
        assert np.array_equal(pos.cpu().numpy(), want["positions"]) and np.array_equal(past.cpu().numpy(), want["context"]) and int(count) == want["left"]
        lens = lens + np.array(step)


@pytest.mark.gpu
@pytest.mark.parametrize("rotary,first,n", [(128, 0, 100), (16, 5, 1), (64, 131000, 300), (96, 2**31 - 40, 40)])
def test_rope_table(rotary, first, n):
    freq = 1e6 ** (-np.arange(rotary // 2) / (rotary // 2))
    t = hma.hma_rope_table(freq, n, first_pos=first, scale=1.25).cpu().numpy().astype(np.float64)
    a = np.arange(first, first + n, dtype=np.float64)[:, None] * freq
    # one rounding to fp32 (half a step, relative), and the 64-bit function's own few 2^-53 beside it
    for got, want in ((t[:, :rotary // 2], 1.25 * np.cos(a)), (t[:, rotary // 2:], 1.25 * np.sin(a))):
        assert (np.abs(got - want) <= 2.0 ** -24 * np.abs(want) * (1 + 1e-6) + 1e-14).all()


def test_arguments_are_checked():
    """Refusals that need no GPU: no cache, tensors that are not on one."""
    L = hma.lib()
    assert L.hma_step_tables(None, None, None, 1, None, 1, None, None, None, None, None, None, 1, None, None) == hma.HMA_ERR_INVALID_ARG
    assert L.hma_release_pages(None, None, None, 1, None, 1, None, None, None) == hma.HMA_ERR_INVALID_ARG
    import ctypes
    d = (ctypes.c_double * 64)()
    for rot, first, n, want in ((8, 0, 1, 2), (24, 0, 1, 2), (144, 0, 1, 2), (64, -1, 1, 1), (64, 0, -1, 1), (64, 2**31, 1, 2), (64, 2**31 - 1, 2, 2), (64, 0, 1, 1), (64, 0, 0, 0)):
        assert L.hma_rope_table(d, rot, first, n, 1.0, None, None) == want, (rot, first, n)
    assert L.hma_rope_table(d, 64, 0, 1, 1.0, 8, None) == hma.HMA_ERR_ALIGNMENT

    class Fake:
        desc, handle = hma.make_desc(1, 8, 8, 4), None
    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(hma.HmaError) as e:
        hma.hma_step_tables(Fake, t, t, t.view(2, 2), t, t, t, t, t, t)
    assert e.value.status == hma.HMA_ERR_INVALID_ARG
    with pytest.raises(hma.HmaError):
        hma.KVCache(Fake.desc, layers=[])
    with pytest.raises(hma.HmaError):
        hma.KVCache(Fake.desc, layers=[torch.zeros(10, dtype=torch.uint8)])


@pytest.mark.gpu
def test_arguments_are_checked_on_the_gpu():
    pool = Pool([4, 4], 4, 3)
    past, table, free, count = pool.gpu()
    i32 = dict(dtype=torch.int32, device="cuda")
    starts, pos, slots = torch.zeros(3, **i32), torch.zeros(4, **i32), torch.zeros(4, dtype=torch.int64, device="cuda")
    good = [past, past, table, free, count, past, starts, pos, slots]
    n0 = hma.hma_launch_count()
    for i, bad in ((0, past.long()), (2, table[:1]), (2, table.t()), (3, free[:2]), (6, starts[:2]), (8, slots[:3]), (8, slots.int())):
        args = list(good)
        args[i] = bad
        with pytest.raises(hma.HmaError):
            hma.hma_step_tables(pool.cache, *args)
    L, p = hma.lib(), lambda t: t.data_ptr()
    for batch, max_pages, max_tokens, want in ((1025, 4, 4, 2), (-1, 4, 4, 1), (2, -1, 4, 1), (2, 4, -1, 1), (2, 1 << 27, 4, 2), (2, 4, (1 << 30) + 1, 2)):
        assert L.hma_step_tables(pool.cache.handle, p(past), p(past), batch, p(table), max_pages, p(free), p(count), p(past), p(starts), p(pos),
                                 p(slots), max_tokens, p(count), None) == want
    assert hma.hma_launch_count() == n0
