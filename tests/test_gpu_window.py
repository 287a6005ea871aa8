"""rkv_window_attention on the GPU against the plain form in 64 bits."""
import pytest
import torch

from tokens_util import TYPES, WIDE, attention, attention_tolerance, descriptor, random_rows, to_pages

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rkv():
    from paper_2505_24133_b200 import build as b
    b.build()
    import paper_2505_24133_b200 as r
    assert r.lib() is not None
    return r


def visible(length, n, window, sinks):
    at = torch.arange(length - n, length, device="cuda")[:, None]
    j = torch.arange(length, device="cuda")[None]
    return (j <= at) & ((at - j < window) | (j < sinks) if window else (j <= at))


class Setup:
    """Rows that no new token sees are NaN, and pages of nothing but such rows have no valid entry in the block table."""

    def __init__(self, rkv, dtype, d, hkv, hq, lens, new, cap, window, sinks, seed=31, paged=False, strided=False, behind=0, offsets=True,
                 longest=None):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.rkv, self.d, self.hkv, self.hq, self.cap = rkv, d, hkv, hq, cap
        self.lens, self.new, self.window, self.sinks = list(lens), list(new), window, sinks
        B, total = len(lens), sum(new) + behind
        self.k, self.v = random_rows((B, hkv, cap, d), dtype, gen), random_rows((B, hkv, cap, d), dtype, gen)
        self.k0, self.v0 = self.k.clone(), self.v.clone()
        unseen = torch.ones(B, cap, dtype=torch.bool, device="cuda")
        for b, (L, n) in enumerate(zip(lens, new)):
            if 0 < n <= L <= cap:
                unseen[b, :L] = ~visible(L, n, window, sinks).any(0)
        mark = 0x7F if dtype == "fp8" else 0xFF
        for x in (self.k, self.v):
            raw = x.view(torch.uint8).view(B, hkv, cap, -1)
            raw[unseen[:, None].expand(B, hkv, cap)] = mark
        self.table = None
        if paged:
            self.k, self.table = to_pages(self.k, gen)
            pool = torch.empty_like(self.k)
            pool.view(torch.uint8).fill_(mark)
            raw = self.v.view(torch.uint8).view(B * hkv * cap // 128, 128, -1)
            pool.view(torch.uint8)[self.table.flatten().long()] = raw
            self.v = pool
            gone = unseen.view(B, 1, cap // 128, 128).all(-1).expand_as(self.table)
            self.table[gone] = -7
        wide = WIDE[dtype]
        rows = torch.randn(total, hq + 3, d, generator=gen, device="cuda").to(wide)
        self.q = rows[:, :hq] if strided else rows[:, :hq].contiguous()
        self.out_rows = torch.full((total, hq + (2 if strided else 0), d), 7.0, device="cuda", dtype=wide)
        self.out = self.out_rows[:, :hq]
        self.seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
        off = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda")
        self.offsets = off if offsets else None
        stride = dict(q_stride=self.q.stride(0), out_stride=self.out.stride(0)) if strided else {}
        self.tokens = rkv.rkv_tokens(total, longest or max(max(new), 1), self.offsets, **stride)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.desc = descriptor(rkv, B, hkv, hq, d, dtype, self.status, self.table, self.k.shape[0] if paged else 0)
        self.workspace(self.desc)

    def workspace(self, desc):
        n = self.rkv.rkv_window_workspace_bytes(desc, self.cap - 1, 1, self.tokens, self.window, self.sinks)
        self.room = torch.full((max(n, 256),), 0xFF, dtype=torch.uint8, device="cuda")
        desc.workspace, desc.workspace_bytes = self.room.data_ptr(), n
        return n

    def call(self, stream=None):
        return self.rkv.rkv_window_attention(self.desc, self.k, self.v, self.q, self.seq, self.out, self.cap - 1, 1, self.tokens, self.window,
                                             self.sinks, stream)

    def check(self, refused=()):
        first, wide = 0, self.out.dtype
        G = self.hq // self.hkv
        for b, (L, n) in enumerate(zip(self.lens, self.new)):
            t = slice(first, first + n)
            first += n
            if b in refused:
                assert (self.out[t] == 0).all()
                continue
            if n == 0:
                continue
            seen = visible(L, n, self.window, self.sinks)
            for h in range(self.hkv):
                ref, size = attention(self.q[t, h * G:(h + 1) * G], self.k0[b, h, :L], self.v0[b, h, :L], seen)
                got = self.out[t, h * G:(h + 1) * G].double()
                assert torch.isfinite(got).all(), (b, h)
                over = float(((got - ref).abs() - attention_tolerance(ref, size, min(L, (self.window or L) + self.sinks), self.d, wide)).max())
                assert over <= 0, (b, h, over)
        assert (self.out[first:] == 7.0).all() and (self.out_rows[:, self.hq:] == 7.0).all()
        assert int(self.status.item()) == (1 if refused else 0)

    def run(self, refused=()):
        assert self.call() == 0
        torch.cuda.synchronize()
        self.check(refused)
        return self


SHAPES = [("bf16", 128), ("bf16", 64), ("bf16", 256), ("fp8", 128), ("fp8", 64), ("f32", 128), ("f32", 64), ("f32", 256)]


@pytest.mark.parametrize("dtype,d", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 3), (100, 4), (128, 0), (129, 128), (300, 130), (4000, 5)])
def test_one_token_per_sequence(rkv, dtype, d, window, sinks):
    """One cached row, lengths on both sides of a tile's and the window's border, a full cache."""
    lens = [1, 2, 127, 128, 129, 300, 431, 640]
    Setup(rkv, dtype, d, 2, 8, lens, [1] * 8, 640, window, sinks, offsets=False).run()


@pytest.mark.parametrize("dtype,d", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4), (300, 130)])
@pytest.mark.parametrize("batch", [4, 90])
def test_one_token_per_sequence_paged(rkv, dtype, d, window, sinks, batch):
    """Pages behind the lengths and outside the windows do not exist, and nothing asks for them."""
    lens = [1, 300, 640, 128] + [(53 * b) % 640 + 1 for b in range(batch - 4)]
    Setup(rkv, dtype, d, 2, 8, lens, [1] * batch, 640, window, sinks, paged=True, offsets=False).run()


@pytest.mark.parametrize("dtype,d", SHAPES)
@pytest.mark.parametrize("window,sinks,paged", [(0, 0, False), (0, 9, True), (1, 1, True), (60, 4, False), (200, 130, True), (257, 0, True)])
def test_ragged_prompts(rkv, dtype, d, window, sinks, paged):
    """Prompts and pieces of prompts of 0 to 300 tokens over caches that hold more, or nothing else."""
    new = [0, 1, 5, 128, 129, 300, 0, 33]
    lens = [0, 1, 400, 128, 640, 300, 50, 513]
    Setup(rkv, dtype, d, 2, 8, lens, new, 640, window, sinks, paged=paged, strided=True, behind=3).run()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp8", 128), ("f32", 128)])
def test_one_token_per_sequence_strided_or_with_gaps(rkv, dtype, d):
    """Queries out of a wider projection; and a batch in which some sequences have no token in the call."""
    Setup(rkv, dtype, d, 2, 6, [5, 200, 300], [1, 1, 1], 384, 100, 4, strided=True, offsets=False).run()
    Setup(rkv, dtype, d, 2, 6, [5, 200, 300, 7], [1, 0, 1, 0], 384, 100, 4, behind=2).run()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp8", 128)])
def test_many_sequences_of_different_lengths(rkv, dtype, d):
    """More items than blocks, most of them with few keys or none."""
    new = [(37 * b) % 210 for b in range(150)]
    lens = [n + (91 * b) % 300 for b, n in enumerate(new)]
    Setup(rkv, dtype, d, 2, 8, lens, new, 512, 150, 4).run()


@pytest.mark.parametrize("hkv,hq", [(1, 1), (3, 3), (2, 6), (1, 5), (2, 12), (1, 7), (2, 16), (1, 16), (1, 48), (1, 100), (1, 130)])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp8", 128), ("f32", 128)])
def test_head_layouts(rkv, dtype, d, hkv, hq):
    Setup(rkv, dtype, d, hkv, hq, [40, 259], [40, 77], 300, 50, 4).run()
    Setup(rkv, dtype, d, hkv, hq, [40, 259], [1, 1], 300, 150, 4, offsets=False).run()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp8", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("n,window,sinks", [(1, 0, 0), (1, 2500, 4), (2, 0, 0), (3, 3000, 200), (40, 0, 0), (700, 1500, 4)])
def test_long_caches(rkv, dtype, d, n, window, sinks):
    """Few rows over many keys: the keys are split between blocks."""
    Setup(rkv, dtype, d, 1, 4, [5000, 4999], [n, n], 5120, window, sinks, offsets=n > 1, paged=True).run()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp8", 128), ("bf16", 64), ("f32", 128)])
def test_long_prompts(rkv, dtype, d):
    """Every piece of a prompt of 1500 tokens, whole and with a window."""
    for window, sinks in ((0, 0), (333, 4)):
        Setup(rkv, dtype, d, 2, 8, [1500, 900], [1500, 900], 1536, window, sinks).run()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp8", 128), ("f32", 128)])
@pytest.mark.parametrize("step", [True, False])
def test_bad_lengths_give_zeros(rkv, dtype, d, step):
    n = 1 if step else 4
    s = Setup(rkv, dtype, d, 2, 4, [-1, 100, 301, n - 1, 300], [n] * 5, 300, 50, 4, offsets=not step)
    s.run(refused=(0, 2, 3))


def test_bad_offsets_write_nothing(rkv):
    s = Setup(rkv, "bf16", 128, 2, 4, [50, 60, 70], [4, 4, 4], 300, 50, 4)
    s.offsets.copy_(torch.tensor([0, 4, 11, 12], dtype=torch.int32))          # more tokens than the call said
    assert s.call() == 0
    torch.cuda.synchronize()
    assert (s.out[4:11] == 7.0).all() and int(s.status.item()) == 1
    assert (s.out[:4] != 7.0).any() and (s.out[11:] != 7.0).any()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp8", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("n", [1, 30])
def test_pages_that_do_not_exist_count_as_zeros(rkv, dtype, d, n):
    s = Setup(rkv, dtype, d, 1, 2, [256, 256], [n, n], 256, 0, 0, paged=True)
    s.table[0, 0, 1], s.table[1, 0, 0] = -1, 1 << 30
    assert s.call() == 0
    torch.cuda.synchronize()
    assert int(s.status.item()) == 1
    s.k0.view(torch.uint8)[0, :, 128:] = 0
    s.v0.view(torch.uint8)[0, :, 128:] = 0
    s.k0.view(torch.uint8)[1, :, :128] = 0
    s.v0.view(torch.uint8)[1, :, :128] = 0
    s.status.zero_()
    s.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 128)])
def test_large_scores(rkv, dtype, d):
    """Scores whose exponentials overflow and underflow 32 bits, growing and falling along the cache."""
    for sign in (1.0, -1.0):
        s = Setup(rkv, dtype, d, 1, 4, [700, 640], [200, 1], 700, 0, 0)
        ramp = sign * torch.linspace(-8, 8, 700, device="cuda")
        for x in (s.k, s.k0):
            x.copy_((ramp[:, None] * torch.ones(d, device="cuda")).to(x.dtype).expand_as(x))
        s.q.copy_((s.q.float() * 0.25 + 4.0).to(s.q.dtype))
        assert s.call() == 0
        torch.cuda.synchronize()
        first = 0
        for b, (L, n) in enumerate(zip(s.lens, s.new)):
            # scores up to 8 * 4 * 128 / sqrt(128) = 362 (bf16 products are exact, sums off by 130 * 2^-24 * 362 < 0.003)
            ref, size = attention(s.q[first:first + n], s.k0[b, 0, :L], s.v0[b, 0, :L], visible(L, n, 0, 0))
            tol = (ref.abs() + size) * 2.0 ** -8 * (1 if dtype == "bf16" else 0) + size * 2 * (0.003 + 2.0 ** -12)
            assert torch.isfinite(s.out[first:first + n]).all()
            assert ((s.out[first:first + n].double() - ref).abs() <= tol).all()
            first += n


def test_rows_beyond_32_bits(rkv):
    """The last head of a cache of more than 2^31 elements."""
    hkv, cap, d = 20, 1 << 20, 128
    k = torch.zeros(1, hkv, cap, d, dtype=torch.float8_e4m3fn, device="cuda")
    v = torch.zeros_like(k)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for x in (k, v):
        x[0, :, cap - 300:] = torch.randn(hkv, 300, d, generator=gen, device="cuda").to(x.dtype)
    for n in (1, 5):
        q = torch.randn(n, hkv, d, generator=gen, device="cuda").to(torch.bfloat16)
        out = torch.zeros_like(q)
        seq = torch.tensor([cap], dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        desc = descriptor(rkv, 1, hkv, hkv, d, "fp8", status)
        tokens = rkv.rkv_tokens(n, n)
        room = torch.empty(rkv.rkv_window_workspace_bytes(desc, cap - 1, 1, tokens, 200, 0) or 256, dtype=torch.uint8, device="cuda")
        desc.workspace, desc.workspace_bytes = room.data_ptr(), room.numel()
        assert rkv.rkv_window_attention(desc, k, v, q, seq, out, cap - 1, 1, tokens, 200, 0) == 0
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        seen = visible(cap, n, 200, 0)[:, cap - 300:]
        for h in range(hkv):
            ref, size = attention(q[:, h:h + 1], k[0, h, cap - 300:].float(), v[0, h, cap - 300:].float(), seen)
            assert ((out[:, h:h + 1].double() - ref).abs() <= attention_tolerance(ref, size, 200, d, torch.bfloat16)).all(), h


def test_another_stream_and_captured_graphs(rkv):
    """Two captured calls of different shapes that share a workspace, replayed in turn, give what eager calls gave."""
    a = Setup(rkv, "bf16", 128, 2, 8, [900, 800], [1, 1], 1024, 0, 0, offsets=False)
    c = Setup(rkv, "bf16", 128, 2, 8, [900, 800], [40, 7], 1024, 300, 4, seed=32)
    n = max(a.room.numel(), c.room.numel())
    room = torch.empty(n, dtype=torch.uint8, device="cuda")
    for x in (a, c):
        x.desc.workspace, x.desc.workspace_bytes = room.data_ptr(), n
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for x in (a, c):
        assert x.call(side) == 0
    torch.cuda.synchronize()
    a.check(), c.check()
    want = a.out.clone(), c.out.clone()
    graphs = []
    for x in (a, c):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            assert x.call() == 0
        graphs.append(g)
    for _ in range(2):
        a.out.zero_(), c.out.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want[0]) and torch.equal(c.out, want[1])


def test_append_then_attend_like_a_decode_loop(rkv):
    """A prompt, three decode steps and a compression: after each append the attention sees the rows that are there, rotated."""
    from tokens_util import rotation_table
    B, hkv, hq, d, budget, buffer, alpha = 2, 2, 8, 128, 128, 64, 8
    cap = budget + buffer
    comp = rkv.Compressor(B, hkv, hq, budget, buffer, alpha)
    gen = torch.Generator(device="cuda").manual_seed(33)
    draw = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    k, v = (torch.full((B, hkv, cap, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    seq = torch.zeros(B, dtype=torch.int32, device="cuda")
    position = torch.zeros(B, dtype=torch.int32, device="cuda")
    table = rotation_table(1024, d)
    prompts = [189, 150]
    q_window = draw(B, hq, alpha, d)

    def step(tokens, counts):
        n = tokens.total
        kn, vn, qn = draw(n, hkv, d), draw(n, hkv, d), draw(n, hq, d)
        q, out = torch.empty_like(qn), torch.empty_like(qn)
        assert rkv.rkv_append_rotary(comp.desc, k, v, kn, vn, seq, budget, buffer, tokens, rkv.rkv_rotary(table, d, position), qn, q) == 0
        position.add_(torch.tensor(counts, dtype=torch.int32, device="cuda"))
        room = torch.empty(rkv.rkv_window_workspace_bytes(comp.desc, budget, buffer, tokens, 100, 4) or 256, dtype=torch.uint8, device="cuda")
        desc = descriptor(rkv, B, hkv, hq, d, "bf16", comp.status)
        desc.workspace, desc.workspace_bytes = room.data_ptr(), room.numel()
        assert rkv.rkv_window_attention(desc, k, v, q, seq, out, budget, buffer, tokens, 100, 4) == 0
        torch.cuda.synchronize()
        comp.check_status()
        first = 0
        for b, m in enumerate(counts):
            L = int(seq[b])
            for h in range(hkv):
                heads = slice(h * 4, h * 4 + 4)
                ref, size = attention(q[first:first + m, heads], k[b, h, :L], v[b, h, :L], visible(L, m, 100, 4))
                over = (out[first:first + m, heads].double() - ref).abs() - attention_tolerance(ref, size, 104, d, torch.bfloat16)
                assert float(over.max()) <= 0
            first += m

    step(rkv.rkv_tokens(sum(prompts), max(prompts), torch.tensor([0, 189, 339], dtype=torch.int32, device="cuda")), prompts)
    for _ in range(3):
        step(rkv.rkv_tokens(B, 1), [1, 1])
    assert seq.tolist() == [192, 153]
    comp.compress(k, v, q_window, seq)
    torch.cuda.synchronize()
    comp.check_status()
    assert seq.tolist() == [budget, budget] and position.tolist() == [192, 153]
    step(rkv.rkv_tokens(B, 1), [1, 1])                       # positions go on where they were, rows where the compression left them
    assert seq.tolist() == [budget + 1, budget + 1] and position.tolist() == [193, 154]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp8", 128), ("f32", 128)])
def test_two_prompts_at_once(rkv, dtype, d):
    """Calls with workspaces of their own on two streams, each of more items than the GPU takes at a time, give what they give one after the other."""
    a = Setup(rkv, dtype, d, 2, 8, [900, 500, 70], [900, 500, 70], 1024, 0, 0, seed=44)
    b = Setup(rkv, dtype, d, 2, 8, [1000, 30, 640], [1000, 30, 600], 1024, 200, 4, seed=45)
    for s in (a, b):
        assert s.call() == 0
    torch.cuda.synchronize()
    want = a.out.clone(), b.out.clone()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    a.out.zero_(), b.out.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for s, st in zip((a, b), streams):
            assert s.call(st) == 0
    torch.cuda.synchronize()
    assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])
    a.check(), b.check()


def test_a_generous_bound_on_the_tokens(rkv):
    """`longest` far above what any sequence has costs time, not results."""
    Setup(rkv, "bf16", 128, 2, 8, [40, 259, 7], [40, 77, 0], 300, 50, 4, longest=20000).run()
    Setup(rkv, "f32", 64, 2, 8, [40, 259, 7], [40, 77, 0], 300, 50, 4, longest=5000).run()


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (55, 3), (56, 56), (57, 130), (128, 4), (200, 129)])
@pytest.mark.parametrize("batch", [9, 160])
def test_single_tokens_of_32_bits_copy_their_rows_in_runs(rkv, batch, window, sinks, paged):
    """The first rows' end, the window's start and the pages' ends fall at every place of a tile, in calls that split the rows and in calls that do not."""
    lens = [1 + (53 * b) % 400 for b in range(batch - 3)] + [384, 128, 1]
    Setup(rkv, "f32", 128, 2, 6, lens, [1] * batch, 512, window, sinks, offsets=False, paged=paged).run()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp8", 128)])
@pytest.mark.parametrize("G,new", [(4, [1500, 900]), (7, [1100, 1033]), (4, [20, 11])])
def test_maxima_that_move_between_the_halves_of_a_tile(rkv, dtype, d, G, new):
    """Keys whose size changes every 64 rows: the maximum is now in one thread's half of a row's keys, now in the other's, and each has to take
    it from the other at every tile.  The same to the bit whenever it is called."""
    s = Setup(rkv, dtype, d, 2, 2 * G, [1500, 1100], new, 1536, 0, 0)
    size = torch.tensor([0.25, 1.0, 2.0, 0.5, 0.25, 2.0, 1.0], device="cuda")[torch.arange(1536, device="cuda") // 64 % 7]
    for x in (s.k, s.k0):
        x.copy_((x.float() * size[:, None]).to(x.dtype))
    assert s.call() == 0
    torch.cuda.synchronize()
    first = 0
    for b, (L, n) in enumerate(zip(s.lens, s.new)):
        for h in range(s.hkv):
            heads = slice(h * G, (h + 1) * G)
            ref, mean = attention(s.q[first:first + n, heads], s.k0[b, h, :L], s.v0[b, h, :L], visible(L, n, 0, 0))
            # keys up to twice as long as those that attention_tolerance counts on: its scores' part once more
            tol = attention_tolerance(ref, mean, L, d, s.out.dtype) + mean * 2 * (d + 2) * 2.0 ** -24 * 2 * d ** 0.5
            assert ((s.out[first:first + n, heads].double() - ref).abs() <= tol).all()
        first += n
    want = s.out.clone()
    for _ in range(30):
        s.out.zero_()
        assert s.call() == 0
        torch.cuda.synchronize()
        assert torch.equal(s.out, want)


def shared_pages(dtype, d, heads, cap, gen, pages=500):
    """Pools of pages that all heads' tables draw from (the attention only reads them), so that long caches of many heads take little room: pool of K,
    of V, table [heads, cap / 128]."""
    pools = [torch.randn(pages, 128, d, generator=gen, device="cuda").to(TYPES[dtype]) for _ in range(2)]
    table = torch.stack([torch.randperm(pages, generator=gen, device="cuda")[:cap // 128] for _ in range(heads)])
    return pools[0], pools[1], table.to(torch.int32)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp8", 128), ("f32", 128), ("fp8", 64)])
@pytest.mark.parametrize("B,cap,window,sinks", [(9, 30848, 0, 0), (5, 57344, 0, 0), (8, 57344, 35000, 200)])
def test_single_tokens_over_long_caches_of_many_heads(rkv, dtype, d, B, cap, window, sinks):
    """The keys of a head are split between more blocks than a cluster has."""
    gen, hkv, G = torch.Generator(device="cuda").manual_seed(61), 8, 2
    k, v, table = shared_pages(dtype, d, B * hkv, cap, gen)
    lens = [cap, 1, cap - 77, 200, cap - 128, 15000, 129, cap, 128][:B]
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q = torch.randn(B, hkv * G, d, generator=gen, device="cuda").to(WIDE[dtype])
    out, status = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = descriptor(rkv, B, hkv, hkv * G, d, dtype, status, table, k.shape[0])
    tokens = rkv.rkv_tokens(B, 1)
    n = rkv.rkv_window_workspace_bytes(desc, cap - 1, 1, tokens, window, sinks)
    room = torch.full((max(n, 256),), 0xFF, dtype=torch.uint8, device="cuda")
    desc.workspace, desc.workspace_bytes = room.data_ptr(), n
    assert rkv.rkv_window_attention(desc, k, v, q, seq, out, cap - 1, 1, tokens, window, sinks) == 0
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for b, L in enumerate(lens):
        seen = visible(L, 1, window, sinks)
        for h in range(hkv):
            rows = table[b * hkv + h].long()
            keys, values = (x[rows].float().view(cap, d)[:L] for x in (k, v))
            ref, size = attention(q[b:b + 1, h * G:(h + 1) * G], keys, values, seen)
            over = (out[b:b + 1, h * G:(h + 1) * G].double() - ref).abs() - attention_tolerance(ref, size, L, d, q.dtype)
            assert float(over.max()) <= 0, (b, h)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp8", 128), ("fp8", 64), ("f32", 128)])
@pytest.mark.parametrize("B,hkv,G,cap", [(3, 2, 4, 128), (2, 1, 8, 640), (40, 8, 1, 1920), (30, 8, 3, 3584)])
def test_many_small_weights_beside_one_that_counts_for_nothing(rkv, dtype, d, B, hkv, G, cap):
    """One row takes nearly all the weight, and its values are zeros: the output is made of the weights of all other rows, 2^-8 to 2^-30 of the
    largest, and each of them is held as well as a large one."""
    key = lambda x: torch.tensor(x, device="cuda").to(TYPES[dtype])                # noqa: E731
    for k in (0.5, 0.125, 0.0, -0.125, -0.25, -0.375, -0.5, -0.625, -0.75):          # weights 2^(-1.443 sqrt(d) (1 - k)) of the largest
        lens = [cap - 28 - b for b in range(B)]
        s = Setup(rkv, dtype, d, hkv, hkv * G, lens, [1] * B, cap, 0, 0, offsets=False)
        for x, other in ((s.k, s.v), (s.k0, s.v0)):
            for b, L in enumerate(lens):
                x[b, :, :L] = key(k)
                x[b, :, 5] = key(1.0)
                other[b, :, :L] = (other[b, :, :L].float() + 1.0).to(other.dtype)
                other[b, :, 5] = key(0.0)
        s.q.fill_(1.0)
        assert s.call() == 0
        torch.cuda.synchronize()
        assert int(s.status.item()) == 0
        for b in {0, B // 2, B - 1}:
            L = lens[b]
            for h in range(hkv):
                ref, size = attention(s.q[b:b + 1, h * G:(h + 1) * G], s.k0[b, h, :L], s.v0[b, h, :L], visible(L, 1, 0, 0))
                # |q| |k| = d at most, values up to 1 larger: within what attention_tolerance counts on, whose `size` is that of these values
                over = (s.out[b:b + 1, h * G:(h + 1) * G].double() - ref).abs() - attention_tolerance(ref, size, L, d, s.out.dtype)
                assert float(over.max()) <= 0, (k, b, h, float((over / size).max()))


@pytest.mark.parametrize("dtype,d", SHAPES)
@pytest.mark.parametrize("window,paged", [(0, False), (30, True)])
def test_values_that_a_token_does_not_see_count_for_nothing(rkv, dtype, d, window, paged):
    """Rows that other tokens of the call see, with values as large as the type has them: not a bit of the tokens that do not see them changes."""
    s = Setup(rkv, dtype, d, 2, 8, [100, 300, 640], [100, 150, 33], 640, window, 0, paged=paged).run()
    want = s.out.clone()
    late = torch.zeros(640, dtype=torch.bool, device="cuda")
    late[[60, 200, 222, 260, 627, 636]] = True
    rows = late.view(1, 1, 640, 1).expand(3, 2, 640, d)
    most = torch.full_like(rows, 0x7E if dtype == "fp8" else 1, dtype=torch.uint8)
    most = most.view(TYPES[dtype]) if dtype == "fp8" else torch.full_like(rows, torch.finfo(TYPES[dtype]).max, dtype=TYPES[dtype])
    if paged:
        mine = s.table.clamp_min(0).long()                   # (pages that nobody sees have no entry)
        for page, spot in zip(mine.flatten(), rows.reshape(-1, 128, d)):
            s.v[page] = torch.where(spot, most.reshape(-1, 128, d)[0], s.v[page])
    else:
        s.v.copy_(torch.where(rows, most, s.v))
    assert s.call() == 0
    torch.cuda.synchronize()
    first, blind = 0, 0
    for b, (L, n) in enumerate(zip(s.lens, s.new)):
        sees = (visible(L, n, window, 0) & late[:L]).any(1)
        for t in torch.nonzero(~sees).flatten().tolist():
            assert torch.equal(s.out[first + t], want[first + t]), (b, t)
            blind += 1
        first += n
    assert blind >= 60


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype,d", SHAPES)
@pytest.mark.parametrize("hkv,G,lens,new,cap,window", [
    (2, 4, [300, 64, 640], [1, 1, 1], 640, 0), (8, 4, [200 + b for b in range(40)], [1] * 40, 300, 100),      # single tokens, split and not
    (1, 2, [5000, 4999], [1, 1], 5120, 0), (1, 2, [5000, 4999], [2, 3], 5120, 0),                             # few rows over many keys
    (2, 4, [300, 400], [100, 37], 640, 150), (8, 4, [700, 600, 650], [500, 600, 333], 720, 0)])               # prompts
def test_a_query_that_is_no_number_gives_none(rkv, value, dtype, d, hkv, G, lens, new, cap, window):
    """NaN for that token and head however the call is cut into blocks, and nothing else changes.  (An infinity: every score is infinite, of either
    sign, or NaN.)"""
    s = Setup(rkv, dtype, d, hkv, hkv * G, lens, new, cap, window, 0, offsets=max(new) > 1).run()
    want, total = s.out.clone(), sum(new)
    hit = [(0, 1), (total - 1, hkv * G - 1), (total // 2, 0)]
    for t, h in hit:
        s.q[t, h, (7 * t + 3) % d] = value
    assert s.call() == 0
    torch.cuda.synchronize()
    assert int(s.status.item()) == 0
    for t, h in hit:
        assert s.out[t, h].isnan().all(), (t, h)
        s.out[t, h] = want[t, h]
    assert torch.equal(s.out, want)


@pytest.mark.parametrize("dtype,d", SHAPES)
@pytest.mark.parametrize("lens,new,window", [([700, 640], [200, 1], 0), ([700, 640], [350, 100], 300), ([700, 1, 640], [1, 1, 1], 0), ([700] * 40, [1] * 40, 0)])
@pytest.mark.parametrize("way", ["up", "down", "peak", "valley"])
def test_large_scores_in_every_form(rkv, dtype, d, lens, new, window, way):
    """Scores between -370 and 370 that grow, fall, or turn inside the cache: maxima that move at every tile or never again, exponentials from far below
    the smallest number to the reference of the weights and beyond it; prompts, pieces of prompts and single tokens."""
    s = Setup(rkv, dtype, d, 1, 4, lens, new, 700, window, 0, offsets=max(new) > 1)
    x = torch.linspace(-8, 8, 700, device="cuda")
    ramp = {"up": x, "down": -x, "peak": 8 - 2 * x.abs(), "valley": 2 * x.abs() - 8}[way] * (128 / d) ** 0.5
    for k in (s.k, s.k0):
        k.copy_(ramp[:, None].expand(700, d).to(k.dtype).expand_as(k))
    s.q.copy_((s.q.float() * 0.25 + 4.0).to(s.q.dtype))
    assert s.call() == 0
    torch.cuda.synchronize()
    assert int(s.status.item()) == 0
    first = 0
    for b, (L, n) in enumerate(zip(s.lens, s.new)):
        ref, size = attention(s.q[first:first + n], s.k0[b, 0, :L], s.v0[b, 0, :L], visible(L, n, window, 0))
        # products of 8-bit or bf16 factors are exact; scores up to 8 * (4 + 4 * 0.25 / d ** 0.5) * 128 ** 0.5 < 400, their sums off by (d + 2) 2^-24
        # of that, of 32-bit factors by as much again; then the factor log2(e) / sqrt(d) and the difference from the maximum, each a rounding of at
        # most 600 in base 2: 4 * 600 * 2^-24 in all.  Twice that for numerator and denominator, 2^-12 for the exponentials, bf16 weights, the output.
        off = 2 * (d + 2) * 2.0 ** -24 * 400 + 4 * 600 * 2.0 ** -24
        tol = (ref.abs() + size) * 2.0 ** -8 * (0 if dtype == "f32" else 1) + size * 2 * (off + 2.0 ** -12)
        got = s.out[first:first + n].double()
        assert torch.isfinite(got).all() and ((got - ref).abs() <= tol).all(), (b, float(((got - ref).abs() - tol).max()))
        first += n


@pytest.mark.parametrize("dtype,d", SHAPES)
@pytest.mark.parametrize("new", [[1, 1, 1], [100, 64, 37]])
def test_windows_and_sinks_up_to_the_largest_number(rkv, dtype, d, new):
    """They see all rows up to the token's own, as window 0 does."""
    most = 2 ** 31 - 1
    for window, sinks in ((most, 0), (most, most), (1, most), (most - 1, 5), (650, most)):
        s = Setup(rkv, dtype, d, 2, 8, [300, 100, 640], new, 640, 0, 0, offsets=max(new) > 1)
        s.window, s.sinks = window, sinks
        s.workspace(s.desc)
        assert s.call() == 0
        torch.cuda.synchronize()
        s.window, s.sinks = 0, 0
        s.check()


@pytest.mark.parametrize("dtype,d", SHAPES)
@pytest.mark.parametrize("lens,new", [([300, 64, 640], [1, 1, 1]), ([300, 64, 640], [100, 64, 37]), ([5000, 4999], [3, 2])])
@pytest.mark.parametrize("paged", [False, True])
def test_captured_calls_of_every_type(rkv, dtype, d, lens, new, paged):
    """Three calls in one graph, whose kernels start early beside one another and share the workspace."""
    s = Setup(rkv, dtype, d, 2, 8, lens, new, 5120 if max(lens) > 640 else 640, 0, 0, offsets=max(new) > 1, paged=paged).run()
    want = s.out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        for _ in range(3):
            assert s.call() == 0
    for _ in range(3):
        s.out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s.out, want)
