"""Pages of the paged cache (fluxbin_pages_resize, fluxbin_pages_fork, fluxbin_kv8_copy_pages) against plain loops, exactly,
and a serving loop that uses them with rotations, drafted trees and kept rows, eager and captured."""
import numpy as np
import pytest

from oracle import quant_oracle as qo
from oracle import serve_oracle as so

from conftest import gpu_available
from gpu_util import log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def fb():
    if not gpu_available():
        pytest.skip("no GPU")
    from paper_2608_15602_amd import fluxbin
    fluxbin.lib()
    return fluxbin


class Pages:
    def __init__(self, fb, pages, P, B, blocks, stride=None):
        import torch
        self.fb, self.torch, self.plain = fb, torch, so.Pool(pages, P)
        self.pool = fb.make_page_pool(pages, P)
        self.table = np.full((B, blocks), -1, np.int32)
        self.wide = torch.full((B, stride or blocks + 3), -9, dtype=torch.int32, device="cuda")
        self.t = self.wide[:, :blocks]
        self.t.fill_(-1)

    def ints(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()

    def check(self):
        assert np.array_equal(self.pool.refs.cpu().numpy(), self.plain.refs)
        assert int(self.pool.missing) == self.plain.missing
        assert np.array_equal(self.t.cpu().numpy(), self.table) and (self.wide[:, self.t.shape[1]:] == -9).all()
        low = int(self.pool.state[0])
        assert 0 <= low <= len(self.plain.refs) and (self.plain.refs[:low] > 0).all() and int(self.pool.state[2]) == 0

    def resize(self, tokens):
        self.fb.fluxbin_pages_resize(self.pool, self.t, self.ints(tokens))
        self.plain.resize(self.table, tokens)
        self.check()

    def fork(self, context, source, blocks, columns=None):
        child = np.full((len(source), blocks), 5, np.int32)
        t = self.ints(child)
        copies = self.fb.fluxbin_pages_fork(self.pool, self.t, self.ints(context), self.ints(source), t)
        want = self.plain.fork(self.table, context, source, child)
        assert np.array_equal(copies.cpu().numpy(), want) and np.array_equal(t.cpu().numpy(), child)
        self.check()
        return t, child


@pytest.mark.parametrize("pages,P,B,blocks", [(7, 16, 2, 4), (100, 64, 5, 30), (5000, 16, 40, 200), (20000, 32, 1500, 12), (4100, 256, 3, 2000)])
def test_resize(fb, pages, P, B, blocks):
    """Random growth and release, past the pool's pages and the table's columns."""
    log(f"case resize pages={pages} B={B} blocks={blocks}")
    s, rng = Pages(fb, pages, P, B, blocks), np.random.default_rng(pages)
    now = np.zeros(B, np.int64)
    for step in range(12):
        kind = step % 4
        if kind == 0:
            now = rng.integers(0, min(blocks * P, 3 * pages * P // B) + 1, B)
        elif kind == 1:
            now = np.maximum(now + rng.integers(-2 * P, 2 * P, B), 0)
        elif kind == 2:
            now = now + 1
        else:
            now = np.where(rng.random(B) < 0.5, -1, rng.integers(0, blocks * P + 2 * P, B))
        s.resize(now)
    s.resize(np.full(B, 2 ** 31 - 1))
    s.resize(np.zeros(B, np.int64))
    assert (s.plain.refs == 0).all()


def test_many_rows_and_pages(fb):
    """More rows than the workgroup that takes pages has threads, of a pool that it looks through in many rounds, on another
    stream, and captured."""
    import torch
    log("case many rows and pages")
    s = Pages(fb, 150000, 16, 2500, 70)
    s.pool.refs[::2] = 1          # pages of others, so that free ones are far apart
    s.plain.refs[::2] = 1
    rng = np.random.default_rng(5)
    s.resize(rng.integers(0, 70 * 16, 2500))
    tokens, side = s.ints(np.zeros(2500)), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fb.fluxbin_pages_resize(s.pool, s.t, tokens)
    for i in range(4):
        want = rng.integers(-50, 70 * 16, 2500)
        tokens.copy_(s.ints(want))
        torch.cuda.synchronize()
        if i % 2:
            fb.fluxbin_pages_resize(s.pool, s.t, tokens, stream=side)
        else:
            graph.replay()
        torch.cuda.synchronize()
        s.plain.resize(s.table, want)
        s.check()


@pytest.mark.parametrize("B,blocks", [(40, 1 << 20), (1100, 1 << 16), (1024, (1 << 21) + (1 << 15)), (1030, 1 << 22)])
def test_wants_past_32_bits(fb, B, blocks):
    """Rows that want 2^25 pages together, and 2^31, and 2^32, up to 1024 rows and more: what there is goes to the first of them,
    and what is missing is counted, up to 2^31 - 1."""
    import torch
    log(f"case wants past 32 bits B={B} blocks={blocks}")
    pool = fb.make_page_pool(64, 16)
    pool.refs[10] = 1
    table = torch.full((B, blocks), -1, dtype=torch.int32, device="cuda")
    tokens = np.full(B, 2 ** 31 - 1, np.int32)
    tokens[:4] = 40, 0, 16 * 30, -1
    wanted = sum(min(-(-int(t) // 16), blocks) for t in tokens[tokens > 0])
    assert wanted > 2 ** 25
    fb.fluxbin_pages_resize(pool, table, torch.from_numpy(tokens).cuda())
    free = [p for p in range(64) if p != 10]
    want = np.full((B, 64), -1, np.int32)
    want[0, :3], want[2, :30], want[4, :30] = free[:3], free[3:33], free[33:]
    assert np.array_equal(table[:, :64].cpu().numpy(), want) and int(table[:, 64:].max()) == -1
    assert (pool.refs == 1).all() and int(pool.missing) == min(wanted - 63, 2 ** 31 - 1)
    fb.fluxbin_pages_resize(pool, table, torch.zeros(B, dtype=torch.int32, device="cuda"))
    assert int(table.max()) == -1 and int(pool.missing) == 0 and pool.refs.nonzero().flatten().tolist() == [10]
    del table
    torch.cuda.empty_cache()


@pytest.mark.parametrize("pages,P,B,C,blocks", [(60, 16, 1, 4, 10), (900, 64, 7, 33, 20), (9000, 32, 30, 1100, 130)])
def test_fork(fb, pages, P, B, C, blocks):
    """Forks that share and copy, forks of forks, pools that run out, sources that are none, narrower and wider tables."""
    log(f"case fork pages={pages} B={B} C={C}")
    s, rng = Pages(fb, pages, P, B, blocks), np.random.default_rng(pages)
    context = rng.integers(0, min(blocks * P, pages * P // (2 * B)), B)
    context[-1] = context[-1] // P * P
    s.resize(context)
    rest = []
    for width in (blocks, blocks + 9, max(1, blocks // 2)):
        source = rng.integers(-1, B + 1, C)
        rest.append(s.fork(context, source, width))
    held = np.array([2 ** 30 if i % 2 else 3 for i in range(B)])
    rest.append(s.fork(held, rng.integers(0, B, C), blocks))       # lengths past what the rows hold
    for t, child in rest:                                          # the children go, in another order than they came
        fb.fluxbin_pages_resize(s.pool, t, s.ints(np.zeros(len(child))))
        s.plain.resize(child, np.zeros(len(child), int))
        assert (t == -1).all()
        s.check()
    s.resize(np.zeros(B, int))
    assert (s.plain.refs == 0).all()


def test_references_of_the_caller(fb):
    log("case references of the caller")
    s = Pages(fb, 20, 16, 2, 8)
    s.pool.refs[:3] += 1
    s.plain.refs[:3] += 1
    s.resize([40, 20])
    assert s.table[0, 0] == 3
    s.pool.refs[1] -= 1
    s.plain.refs[1] -= 1
    s.pool.state[0] = 0
    s.resize([60, 20])
    assert s.table[0, 3] == 1


@pytest.mark.parametrize("P,H,D", [(16, 1, 64), (64, 8, 128), (256, 3, 256)])
def test_copy_pages(fb, P, H, D):
    """Codes and scales, inside a cache and from another of another size; pairs that are none are left out."""
    import torch
    log(f"case copy P={P} H={H} D={D}")
    rng = np.random.default_rng(P)
    a, b = fb.make_kv8_cache(30, P, H, D), fb.make_kv8_cache(11, P, H, D)
    for c in (a, b):
        c.buf.copy_(torch.from_numpy(rng.integers(0, 256, c.buf.numel(), dtype=np.uint8)))
    def parts(cache, pages):
        raw, n = cache.buf.cpu().numpy(), pages * H * P * D
        up = -(-pages * H * 4 // 256) * 256
        return [raw[:n].reshape(pages, -1).copy(), raw[n:2 * n].reshape(pages, -1).copy(),
                raw[2 * n:2 * n + pages * H * 4].reshape(pages, -1).copy(), raw[2 * n + up:2 * n + up + pages * H * 4].reshape(pages, -1).copy()]
    pairs = [(3, 7), (-1, 2), (5, 30), (30, 1), (0, 28), (4, 4), (29, 9), (2 ** 31 - 1, 3), (6, -2 ** 31)]
    x = parts(a, 30)
    fb.fluxbin_kv8_copy_pages(a, torch.tensor(pairs, dtype=torch.int32, device="cuda"))
    for side in x:
        for f, t in pairs:
            if 0 <= f < 30 and 0 <= t < 30:
                side[t] = side[f]
    assert all(np.array_equal(u, v) for u, v in zip(x, parts(a, 30)))
    pairs = [(29, 0), (3, 10), (11, 11), (5, 9)]
    y = parts(b, 11)
    fb.fluxbin_kv8_copy_pages(b, torch.tensor(pairs, dtype=torch.int32, device="cuda"), source_cache=a)
    for u, v in zip(x, y):
        v[0], v[10], v[9] = u[29], u[3], u[5]
    assert all(np.array_equal(u, v) for u, v in zip(y, parts(b, 11)))
    assert all(np.array_equal(u, v) for u, v in zip(x, parts(a, 30)))


def test_refusals(fb):
    import torch
    log("case pages refusals")
    s = Pages(fb, 20, 16, 2, 8)
    one, child = s.ints([1, 1]), s.ints(np.zeros((3, 8)))
    for t, n in ((s.t.long(), one), (s.t.cpu(), one), (s.t.t(), one), (s.t, one[:1]), (s.t, one.long()), (s.t, s.ints([1, 1, 1]))):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_pages_resize(s.pool, t, n)
    for ctx, src, to, copies in ((one[:1], s.ints([0, 0, 0]), child, None), (one, s.ints([0, 0]), child, None), (one, s.ints([0, 0, 0]), child.t(), None),
                                 (one, s.ints([0, 0]), s.t, None), (one, s.ints([0, 0, 0]), child, s.ints([[0, 0]])),
                                 (one, s.ints([0, 0, 0]), child, torch.zeros(3, 2, dtype=torch.int64, device="cuda"))):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_pages_fork(s.pool, s.t, ctx, src, to, copies=copies)
    cache, other = fb.make_kv8_cache(20, 16, 2, 64), fb.make_kv8_cache(20, 16, 4, 64)
    good = s.ints([[1, 2]])
    for c, kw in ((good.long(), {}), (good[0], {}), (good.cpu(), {}), (s.ints([[1, 2, 3]]), {}), (good, dict(source_cache=other))):
        with pytest.raises(fb.FluxbinError):
            fb.fluxbin_kv8_copy_pages(cache, c, **kw)
    s.check()


# ---------------------------------------------------------------------------------------------- as they are used together

class Loop:
    """Speculative decoding of B sequences: pages for the drafted rows, their masks and positions, q and k rotated, rows into
    the cache, attention, the accepted path kept, pages back."""
    HQ, H, D, P, R = 8, 2, 64, 16, 32

    def __init__(self, fb, B, n, pages, blocks, seed):
        import torch
        self.fb, self.torch, self.B, self.n = fb, torch, B, n
        self.rng = np.random.default_rng(seed)
        z = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device="cuda")
        self.cache, self.pool = fb.make_kv8_cache(pages, self.P, self.H, self.D), fb.make_page_pool(pages, self.P)
        self.cache.buf.fill_(0xFF)
        self.table = torch.full((B, blocks), -1, dtype=torch.int32, device="cuda")
        freq = (10000.0 ** (-np.arange(self.R // 2) / (self.R // 2))).astype(np.float32)
        w = (1 + 0.2 * self.rng.standard_normal(self.D)).astype(np.float32)
        self.freq, self.w = freq, w
        self.rotary = fb.make_rotary(self.D, torch.from_numpy(freq).cuda(), torch.from_numpy(w).cuda(), torch.from_numpy(w).cuda())
        T = B * n
        self.qkv = z(T, (self.HQ + 2 * self.H) * self.D, dtype=torch.float16)
        self.parents, self.keep, self.kept = z(T), z(T), z(B)
        self.length, self.context = z(B), z(B)
        self.offsets = torch.arange(0, T + 1, n, dtype=torch.int32, device="cuda")
        self.masks, self.positions = z(T, 1, dtype=torch.int64), z(T)
        self.out = z(T, self.HQ, self.D, dtype=torch.float16)
        self.ws = fb.make_kv8_tree_workspace(self.cache, T, B, self.HQ)
        self.plain, self.ppool = so.Kv8(pages, self.P, self.H, self.D), so.Pool(pages, self.P)
        self.ptable, self.plength = np.full((B, blocks), -1, np.int32), np.zeros(B, np.int64)

    def split(self):
        return (t.unflatten(1, (-1, self.D)) for t in self.qkv.split([self.HQ * self.D, self.H * self.D, self.H * self.D], dim=1))

    def step(self):
        fb = self.fb
        q, k, v = self.split()
        self.torch.add(self.length, self.n, out=self.context)
        fb.fluxbin_pages_resize(self.pool, self.table, self.context)
        fb.fluxbin_tree_masks(self.parents, self.offsets, self.context, 1, masks=self.masks, positions=self.positions)
        fb.fluxbin_qk_rotate(self.rotary, q, k, self.positions, q_out=q, k_out=k)
        fb.fluxbin_kv8_append(self.cache, k, v, self.offsets, self.context, self.table)
        fb.fluxbin_kv8_tree_attention(self.cache, q, self.masks, self.offsets, self.context, self.table, out=self.out, workspace=self.ws)
        fb.fluxbin_kv8_keep(self.cache, self.keep, self.kept, self.offsets, self.context, self.table)
        self.torch.add(self.length, self.kept, out=self.length)
        fb.fluxbin_pages_resize(self.pool, self.table, self.length)

    def draft(self):
        """New inputs: rows, trees, and a path of each as what is accepted."""
        rng, n = self.rng, self.n
        self.rows = rng.standard_normal(self.qkv.shape).astype(np.float16)
        self.pparents = (np.floor(rng.random((self.B, n)) * (np.arange(n) + 1)).astype(np.int32) - 1)
        self.pkeep, self.pkept = np.zeros((self.B, n), np.int32), np.zeros(self.B, np.int32)
        for b in range(self.B):
            node, path = int(rng.integers(0, n)), []
            while node >= 0:
                path.append(node)
                node = int(self.pparents[b, node])
            self.pkeep[b, :len(path)], self.pkept[b] = path[::-1], len(path)
        for t, x in ((self.qkv, self.rows), (self.parents, self.pparents.ravel()), (self.keep, self.pkeep.ravel()), (self.kept, self.pkept)):
            t.copy_(self.torch.from_numpy(np.ascontiguousarray(x)))

    def check(self):
        T, n, offsets = self.B * self.n, self.n, np.arange(0, self.B * self.n + 1, self.n)
        context = self.plength + n
        self.ppool.resize(self.ptable, context)
        masks, positions, _ = so.tree_masks(self.pparents.ravel(), offsets, context, 1, T)
        assert np.array_equal(self.masks.cpu().numpy(), so.packed(masks)) and np.array_equal(self.positions.cpu().numpy(), positions)
        q, k, v = (x.reshape(T, -1, self.D) for x in np.split(self.rows, [self.HQ * self.D, (self.HQ + self.H) * self.D], axis=1))
        gq, gk, gv = (t.cpu().numpy() for t in self.split())
        for x, got in ((q, gq), (k, gk)):
            y, size = so.rotate(x, positions, self.freq, self.w)
            assert (np.abs(got.astype(np.float64) - y) <= so.rotate_bound(y, size)).all()
        assert np.array_equal(gv, v)
        self.plain.append(gk, gv, offsets, context, self.ptable)
        ref, mag, big, peak, _ = self.plain.tree_attention(gq, masks, offsets, context, self.ptable, self.D ** -0.5)
        assert (np.abs(self.out.cpu().double().numpy() - ref) <= qo.attention_bound(ref, mag, big, peak, int(context.max()))).all()
        self.plain.keep(self.pkeep.ravel(), self.pkept, offsets, context, self.ptable, T)
        self.plength = self.plength + self.pkept
        self.ppool.resize(self.ptable, self.plength)
        assert np.array_equal(self.table.cpu().numpy(), self.ptable) and np.array_equal(self.length.cpu().numpy(), self.plength)
        assert np.array_equal(self.pool.refs.cpu().numpy(), self.ppool.refs) and int(self.pool.missing) == 0
        self.cached(self.table, self.ptable, self.plength)

    def cached(self, table, ptable, length):
        """Every cached value, bit for bit."""
        offs = np.concatenate([[0], np.cumsum(length)])
        ints = lambda x: self.torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()
        k, v = self.fb.fluxbin_kv8_read(self.cache, ints(offs), ints(length), table, int(offs[-1]))
        pk, pv, _ = self.plain.read(offs, length, ptable, int(offs[-1]))
        assert np.array_equal(k.cpu().numpy(), pk) and np.array_equal(v.cpu().numpy(), pv)


def test_speculative_decoding(fb):
    import torch
    log("case speculative decoding")
    s = Loop(fb, 3, 24, 60, 12, seed=41)
    for _ in range(3):   # eager
        s.draft()
        s.step()
        s.check()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    for _ in range(8):
        s.draft()
        graph.replay()
        torch.cuda.synchronize()
        s.check()


def test_parallel_samples(fb):
    """Samples of a prompt: forked, then decoded apart; what one appends no other sees. Then the prompts go."""
    import torch
    log("case parallel samples")
    s = Loop(fb, 2, 40, 60, 12, seed=42)
    for _ in range(3):
        s.draft()
        s.step()
        s.check()
    C, source = 5, [0, 1, 1, 0, 1]
    ints = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()
    child, pchild = torch.full((C, 12), -1, dtype=torch.int32, device="cuda"), np.full((C, 12), -1, np.int32)
    copies = fb.fluxbin_pages_fork(s.pool, s.table, s.length, ints(source), child)
    pcopies = s.ppool.fork(s.ptable, s.plength, source, pchild)
    fb.fluxbin_kv8_copy_pages(s.cache, copies)
    for f, t in pcopies:
        if f >= 0:
            s.plain.codes[:, t], s.plain.scales[:, t] = s.plain.codes[:, f], s.plain.scales[:, f]
    length = s.plength[source]
    fb.fluxbin_pages_resize(s.pool, s.table, ints([0, 0]))
    s.ppool.resize(s.ptable, [0, 0])
    for i in range(20):
        length = length + 1
        fb.fluxbin_pages_resize(s.pool, child, ints(length))
        s.ppool.resize(pchild, length)
        k, v = (s.rng.standard_normal((C, s.H, s.D)).astype(np.float16) for _ in range(2))
        offs = np.arange(C + 1)
        fb.fluxbin_kv8_append(s.cache, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), ints(offs), ints(length), child)
        s.plain.append(k, v, offs, length, pchild)
    assert np.array_equal(child.cpu().numpy(), pchild) and np.array_equal(s.pool.refs.cpu().numpy(), s.ppool.refs)
    s.cached(child, pchild, length)
    fb.fluxbin_pages_resize(s.pool, child, ints([0] * C))
    assert not s.pool.refs.any()


def test_cut_into_a_shared_page(fb):
    """A sample cut back to a length inside a page that its prompt holds too: forked at that length, then appended to with larger
    scales, it changes nothing of the prompt's, and ends where a fork of the prompt at that length would."""
    import torch
    log("case cut into a shared page")
    s = Loop(fb, 1, 8, 20, 6, seed=43)
    ints = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()

    def append(table, ptable, offs, length, scale):
        k, v = ((s.rng.standard_normal((offs[-1], s.H, s.D)) * scale).astype(np.float16) for _ in range(2))
        fb.fluxbin_kv8_append(s.cache, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), ints(offs), ints(length), table)
        s.plain.append(k, v, offs, length, ptable)

    def fork(table, ptable, context):
        child, pchild = torch.full((1, 6), -1, dtype=torch.int32, device="cuda"), np.full((1, 6), -1, np.int32)
        copies = fb.fluxbin_pages_fork(s.pool, table, ints(context), ints([0]), child)
        fb.fluxbin_kv8_copy_pages(s.cache, copies)
        for f, t in s.ppool.fork(ptable, context, [0], pchild):
            if f >= 0:
                s.plain.codes[:, t], s.plain.scales[:, t] = s.plain.codes[:, f], s.plain.scales[:, f]
        return child, pchild

    def resize(table, ptable, tokens):
        fb.fluxbin_pages_resize(s.pool, table, ints(tokens))
        s.ppool.resize(ptable, tokens)

    resize(s.table, s.ptable, [40])
    append(s.table, s.ptable, [0, 40], [40], 1.0)
    prompt = [x.clone() for x in fb.fluxbin_kv8_read(s.cache, ints([0, 40]), ints([40]), s.table, 40)]
    child, pchild = fork(s.table, s.ptable, [40])
    cut, pcut = fork(child, pchild, [20])
    resize(child, pchild, [0])
    resize(cut, pcut, [27])
    append(cut, pcut, [0, 7], [27], 30.0)
    assert np.array_equal(cut.cpu().numpy(), pcut) and np.array_equal(s.pool.refs.cpu().numpy(), s.ppool.refs)
    assert s.ppool.refs[pcut[0, 0]] == 2 and s.ppool.refs[pcut[0, 1]] == 1
    s.cached(cut, pcut, np.array([27]))
    now = fb.fluxbin_kv8_read(s.cache, ints([0, 40]), ints([40]), s.table, 40)
    assert all(torch.equal(x, y) for x, y in zip(prompt, now))
