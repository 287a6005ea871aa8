"""rkv_prefix_attention on the GPU against the plain form in 64 bits."""
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


class Setup:
    """Rows beyond the lengths are NaN."""

    def __init__(self, rkv, dtype, d, hkv, hq, lens, prefix_lens, cap, rows, seed=41, paged=False):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.rkv, self.d, self.hkv, self.hq, self.cap = rkv, d, hkv, hq, cap
        self.lens, self.plens = list(lens), list(prefix_lens)
        B, n = len(lens), len(prefix_lens)
        self.k, self.v = (random_rows((B, hkv, cap, d), dtype, gen, lens) for _ in range(2))
        self.pk, self.pv = (random_rows((n, hkv, rows, d), dtype, gen, prefix_lens) for _ in range(2))
        self.plain = [x.clone() for x in (self.k, self.v, self.pk, self.pv)]
        self.table = self.ptable = None
        if paged:
            self.k, self.table = to_pages(self.k, gen)
            self.v = self.other_pool(self.plain[1], self.k, self.table)
            self.pk, self.ptable = to_pages(self.pk, gen)
            self.pv = self.other_pool(self.plain[3], self.pk, self.ptable)
        self.q = torch.randn(B, hq, d, generator=gen, device="cuda").to(WIDE[dtype])
        self.out = torch.full_like(self.q, 7.0)
        self.seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.pseq = torch.tensor(prefix_lens, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.desc = descriptor(rkv, B, hkv, hq, d, dtype, self.status, self.table, self.k.shape[0] if paged else 0)
        self.prefix = rkv.rkv_prefix(self.pk, self.pv, self.pseq, self.ptable)
        n = rkv.rkv_prefix_workspace_bytes(self.desc, cap - 1, 1, self.prefix)
        self.room = torch.full((max(n, 256),), 0xFF, dtype=torch.uint8, device="cuda")
        self.desc.workspace, self.desc.workspace_bytes = self.room.data_ptr(), n

    @staticmethod
    def other_pool(x, like, table):
        pool = torch.empty_like(like)
        pool.view(torch.uint8).fill_(0x7F if x.dtype == torch.float8_e4m3fn else 0xFF)
        pool.view(torch.uint8)[table.flatten().long()] = x.contiguous().view(torch.uint8).view(table.numel(), 128, -1)
        return pool

    def call(self, stream=None):
        return self.rkv.rkv_prefix_attention(self.desc, self.k, self.v, self.q, self.seq, self.out, self.cap - 1, 1, self.prefix, stream)

    def check(self, bad=()):
        k, v, pk, pv = self.plain
        G, per = self.hq // self.hkv, len(self.lens) // len(self.plens)
        for b, L in enumerate(self.lens):
            P = self.plens[b // per]
            L = 0 if b in bad else L
            for h in range(self.hkv):
                keys = torch.cat([pk[b // per, h, :P].float(), k[b, h, :L].float()])
                values = torch.cat([pv[b // per, h, :P].float(), v[b, h, :L].float()])
                got = self.out[b:b + 1, h * G:(h + 1) * G].double()
                if P + L == 0:
                    assert (got == 0).all()
                    continue
                ref, size = attention(self.q[b:b + 1, h * G:(h + 1) * G], keys, values, torch.ones(1, P + L, dtype=torch.bool, device="cuda"))
                assert torch.isfinite(got).all(), (b, h)
                over = float(((got - ref).abs() - attention_tolerance(ref, size, P + L, self.d, self.out.dtype)).max())
                assert over <= 0, (b, h, over)
        assert int(self.status.item()) == (1 if bad else 0)

    def run(self, bad=()):
        assert self.call() == 0
        torch.cuda.synchronize()
        self.check(bad)
        return self


SHAPES = [("bf16", 128), ("bf16", 64), ("bf16", 256), ("fp8", 128), ("fp8", 64), ("f32", 128), ("f32", 64), ("f32", 256)]


@pytest.mark.parametrize("dtype,d", SHAPES)
@pytest.mark.parametrize("paged", [False, True])
def test_lengths(rkv, dtype, d, paged):
    """Prefixes of no row, one row and odd lengths; own caches that are empty, hold one row, are full."""
    Setup(rkv, dtype, d, 2, 8, [0, 1, 127, 256, 0, 129, 5, 200], [300, 0, 1, 257], 256, 384, paged=paged).run()


@pytest.mark.parametrize("hkv,hq", [(1, 1), (2, 6), (1, 5), (2, 14), (1, 8), (1, 16), (1, 100), (1, 130)])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp8", 128), ("f32", 128)])
@pytest.mark.parametrize("batch", [1, 3, 50])
def test_head_layouts_and_batches(rkv, dtype, d, hkv, hq, batch):
    """One row of queries up to many row tiles per prefix."""
    Setup(rkv, dtype, d, hkv, hq, [(37 * b) % 300 for b in range(batch)], [333], 300, 400).run()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp8", 128), ("f32", 128)])
@pytest.mark.parametrize("batch,prefixes,rows,cap", [(2, 1, 6000, 200), (16, 2, 5000, 4500), (48, 3, 2000, 1000), (64, 64, 300, 300), (200, 1, 130, 64)])
def test_long_prefixes_and_many_samples(rkv, dtype, d, batch, prefixes, rows, cap):
    Setup(rkv, dtype, d, 2, 8, [(cap * (b + 1)) // batch for b in range(batch)], [max(0, rows - 7 * p) for p in range(prefixes)], cap, rows).run()


def test_bad_lengths_count_as_none(rkv):
    s = Setup(rkv, "bf16", 128, 2, 8, [50, 301, -1, 20], [300], 300, 300)
    s.run(bad=(1, 2))
    s = Setup(rkv, "bf16", 128, 2, 8, [50, 30, 0, 20], [100, 100], 300, 300)
    s.pseq.copy_(torch.tensor([301, -1], dtype=torch.int32))
    s.plens = [0, 0]
    assert s.call() == 0
    torch.cuda.synchronize()
    assert int(s.status.item()) == 1
    s.status.zero_()
    s.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp8", 128), ("f32", 128)])
def test_pages_that_do_not_exist_count_as_zeros(rkv, dtype, d):
    s = Setup(rkv, dtype, d, 1, 4, [200, 256], [256], 256, 256, paged=True)
    s.ptable[0, 0, 0], s.table[1, 0, 1] = s.pk.shape[0], -3
    assert s.call() == 0
    torch.cuda.synchronize()
    assert int(s.status.item()) == 1
    for x in s.plain[:2]:
        x.view(torch.uint8)[1, :, 128:] = 0
    for x in s.plain[2:]:
        x.view(torch.uint8)[0, :, :128] = 0
    s.status.zero_()
    s.check()


def test_one_prefix_equals_each_sequence_with_the_rows_of_its_own(rkv):
    """The same rows stored in front of every sequence's own: the decode attention over them agrees to the rounding of the output and weights."""
    s = Setup(rkv, "bf16", 128, 2, 8, [40, 200, 0], [300], 256, 300).run()
    k, v, pk, pv = s.plain
    cap = 640
    joined = []
    for own, shared in ((k, pk), (v, pv)):
        x = torch.zeros(3, 2, cap, 128, dtype=torch.bfloat16, device="cuda")
        x[:, :, :300] = shared
        for b, L in enumerate(s.lens):
            x[b, :, 300:300 + L] = own[b, :, :L]
        joined.append(x)
    desc = descriptor(rkv, 3, 2, 8, 128, "bf16", s.status)
    room = torch.empty(rkv.rkv_decode_workspace_bytes(desc, cap - 1, 1), dtype=torch.uint8, device="cuda")
    desc.workspace, desc.workspace_bytes = room.data_ptr(), room.numel()
    out = torch.empty(3, 8, 128, device="cuda")
    lens = torch.tensor([300 + L for L in s.lens], dtype=torch.int32, device="cuda")
    assert rkv.rkv_decode_attention(desc, joined[0], joined[1], s.q, lens, out, cap - 1, 1) == 0
    torch.cuda.synchronize()
    # values N(0, 1), at most 500 of them: |v| < 6; the weights' and the output's rounding are half a bf16 step each
    assert float((out - s.out.float()).abs().max()) <= 2.0 ** -8 * (6.0 + 6.0)


def test_another_stream_and_a_captured_graph(rkv):
    s = Setup(rkv, "bf16", 128, 2, 8, [40, 200, 0, 130], [300, 100], 256, 300)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert s.call(side) == 0
    torch.cuda.synchronize()
    s.check()
    want = s.out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        assert s.call() == 0
    for _ in range(2):
        s.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s.out, want)
    # other lengths, the same graph
    s.lens, s.plens = [10, 0, 256, 1], [1, 300]
    s.seq.copy_(torch.tensor(s.lens, dtype=torch.int32))
    s.pseq.copy_(torch.tensor(s.plens, dtype=torch.int32))
    for x, n in ((s.k, s.lens), (s.v, s.lens), (s.pk, s.plens), (s.pv, s.plens)):
        x.normal_()
    s.plain = [x.clone() for x in (s.k, s.v, s.pk, s.pv)]
    graph.replay()
    torch.cuda.synchronize()
    s.check()


def _chain(rkv, wait):
    """Steps of a batch of samples: append, attend over prefix and own rows, attend over a window; with `wait`, each call finished before the next."""
    gen = torch.Generator(device="cuda").manual_seed(51)
    B, hkv, hq, d, cap, rows = 48, 4, 16, 128, 256, 3000
    draw = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    k, v, pk, pv = draw(B, hkv, cap, d), draw(B, hkv, cap, d), draw(2, hkv, rows, d), draw(2, hkv, rows, d)
    seq = torch.tensor([(5 * b) % 200 for b in range(B)], dtype=torch.int32, device="cuda")
    plens = torch.tensor([rows, 2777], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = descriptor(rkv, B, hkv, hq, d, "bf16", status)
    prefix, tokens, rotary = rkv.rkv_prefix(pk, pv, plens), rkv.rkv_tokens(B, 1), rkv.rkv_rotary(None, 0)
    room = torch.full((max(rkv.rkv_prefix_workspace_bytes(desc, cap - 1, 1, prefix), 256),), 0xFF, dtype=torch.uint8, device="cuda")
    assert room.numel() > 256                                # (two kernels and partial results, not one)
    desc.workspace, desc.workspace_bytes = room.data_ptr(), room.numel()
    new = [(draw(B, hkv, d), draw(B, hkv, d), draw(B, hq, d)) for _ in range(12)]
    outs = [(torch.empty(B, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(B, hq, d, dtype=torch.bfloat16, device="cuda")) for _ in new]
    torch.cuda.synchronize()
    for (kn, vn, q), (a, w) in zip(new, outs):
        calls = (lambda: rkv.rkv_append_rotary(desc, k, v, kn, vn, seq, cap - 1, 1, tokens, rotary),
                 lambda: rkv.rkv_prefix_attention(desc, k, v, q, seq, a, cap - 1, 1, prefix),
                 lambda: rkv.rkv_window_attention(desc, k, v, q, seq, w, cap - 1, 1, tokens, 50, 4))
        for call in calls:
            assert call() == 0
            if wait:
                torch.cuda.synchronize()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return [x for pair in outs for x in pair] + [k, v, seq]


def test_steps_one_behind_the_other_equal_steps_with_waiting(rkv):
    """The kernels of a step start early, beside the ones before them; what they compute is what they compute when each waits for the last."""
    want = _chain(rkv, True)
    for _ in range(3):
        for a, b in zip(_chain(rkv, False), want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp8", 128), ("bf16", 64)])
def test_two_calls_at_once(rkv, dtype, d):
    """Calls with workspaces of their own on two streams give what they give one after the other."""
    a = Setup(rkv, dtype, d, 2, 8, [(17 * b) % 250 for b in range(32)], [2000, 1500], 256, 2048, seed=42)
    b = Setup(rkv, dtype, d, 2, 8, [(23 * b) % 250 for b in range(64)], [1800], 256, 2048, seed=43)
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


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("batch,prefixes", [(8, 4), (160, 4), (12, 12)])
def test_rows_of_32_bits_are_copied_in_runs(rkv, batch, prefixes, paged):
    """The prefix's end, the sequence's and the pages' fall at every place of a tile."""
    lens = [(53 * b) % 400 for b in range(batch - 3)] + [384, 0, 1]
    plens = ([55, 57, 128, 300] + [0, 1, 56, 112, 129, 255, 256, 10])[:prefixes]
    Setup(rkv, "f32", 128, 2, 6, lens, plens, 512, 384, paged=paged).run()


def test_long_shared_prefixes_of_32_bits(rkv):
    """So many sequences that the prefix's rows are read once for all, by a kernel of their own."""
    s = Setup(rkv, "f32", 128, 2, 8, [(37 * b) % 300 for b in range(64)], [1500, 1411], 300, 1500)
    assert 64 * 2 * 1500 * 1024 > 160 << 20
    s.run()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp8", 128)])
def test_prefixes_in_front_of_long_caches_of_many_heads(rkv, dtype, d):
    """A prefix for each sequence, read by the blocks that read its own rows; more of them to a head than a cluster has."""
    from test_gpu_window import shared_pages
    gen, B, hkv, G, cap, rows = torch.Generator(device="cuda").manual_seed(62), 9, 8, 2, 20480, 10368
    k, v, table = shared_pages(dtype, d, B * hkv, cap + rows, gen)
    own, shared = table[:, :cap // 128].contiguous(), table[:, cap // 128:].contiguous().view(B, hkv, rows // 128)
    lens, plens = [cap, 0, cap - 77, 200, 1, 15000, 129, cap, 0], [rows, rows - 1, 300, 0, rows, 128, 1, 5000, 0]
    seq, pseq = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, plens))
    q = torch.randn(B, hkv * G, d, generator=gen, device="cuda").to(WIDE[dtype])
    out, status = torch.full_like(q, 7.0), torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = descriptor(rkv, B, hkv, hkv * G, d, dtype, status, own, k.shape[0])
    prefix = rkv.rkv_prefix(k, v, pseq, shared)
    n = rkv.rkv_prefix_workspace_bytes(desc, cap - 1, 1, prefix)
    room = torch.full((max(n, 256),), 0xFF, dtype=torch.uint8, device="cuda")
    desc.workspace, desc.workspace_bytes = room.data_ptr(), n
    assert rkv.rkv_prefix_attention(desc, k, v, q, seq, out, cap - 1, 1, prefix) == 0
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for b, (L, P) in enumerate(zip(lens, plens)):
        for h in range(hkv):
            heads = slice(h * G, (h + 1) * G)
            if L + P == 0:
                assert (out[b, heads] == 0).all()
                continue
            keys, values = (torch.cat([x[shared[b, h].long()].float().view(rows, d)[:P], x[own[b * hkv + h].long()].float().view(cap, d)[:L]])
                            for x in (k, v))
            ref, size = attention(q[b:b + 1, heads], keys, values, torch.ones(1, P + L, dtype=torch.bool, device="cuda"))
            over = (out[b:b + 1, heads].double() - ref).abs() - attention_tolerance(ref, size, P + L, d, q.dtype)
            assert float(over.max()) <= 0, (b, h)


@pytest.mark.parametrize("dtype,d", SHAPES)
@pytest.mark.parametrize("batch,prefixes,rows,cap", [(2, 2, 300, 200), (4, 1, 300, 700), (48, 1, 2000, 300), (200, 1, 4000, 130)])
def test_a_query_that_is_no_number_gives_none(rkv, dtype, d, batch, prefixes, rows, cap):
    """NaN for that sequence and head whether its prefix is read beside its own rows or apart, and nothing else changes."""
    s = Setup(rkv, dtype, d, 2, 8, [(37 * b) % cap for b in range(batch)], [rows] * prefixes, cap, rows).run()
    want = s.out.clone()
    hit = [(0, 1), (batch - 1, 7)]
    for b, h in hit:
        s.q[b, h, 5 + b % 50] = float("nan")
    assert s.call() == 0
    torch.cuda.synchronize()
    assert int(s.status.item()) == 0
    for b, h in hit:
        assert s.out[b, h].isnan().all(), (b, h)
        s.out[b, h] = want[b, h]
    assert torch.equal(s.out, want)


def _mixed_chain(rkv, dtype, d, B, wait):
    """Pieces of prompts and steps of samples in turn, all calls on one workspace; with `wait`, each call finished before the next."""
    from tokens_util import rotation_table
    hkv, hq, cap, rows = 4, 16, 768, 2048
    gen = torch.Generator(device="cuda").manual_seed(52)
    draw = lambda t, *shape: torch.randn(*shape, generator=gen, device="cuda").to(t[dtype])  # noqa: E731
    k, v, pk, pv = draw(TYPES, B, hkv, cap, d), draw(TYPES, B, hkv, cap, d), draw(TYPES, 2, hkv, rows, d), draw(TYPES, 2, hkv, rows, d)
    seq = torch.tensor([(5 * b) % 200 for b in range(B)], dtype=torch.int32, device="cuda")
    plens = torch.tensor([rows, 1777], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = descriptor(rkv, B, hkv, hq, d, dtype, status)
    prefix, rotary, one = rkv.rkv_prefix(pk, pv, plens), rkv.rkv_rotary(rotation_table(1024, 32), 32), rkv.rkv_tokens(B, 1)
    pieces = []
    for i in range(4):
        ends = torch.tensor([(7 * b + i) % 40 for b in range(B)]).cumsum(0).tolist()
        pieces.append(rkv.rkv_tokens(ends[-1], 40, torch.tensor([0] + ends, dtype=torch.int32, device="cuda")))
    need = max([256, rkv.rkv_prefix_workspace_bytes(desc, cap - 1, 1, prefix)] +
               [rkv.rkv_window_workspace_bytes(desc, cap - 1, 1, t, w, 4) for t in pieces + [one] for w in (0, 100)])
    room = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    desc.workspace, desc.workspace_bytes = room.data_ptr(), need

    def calls(t, window, samples):
        n = t.total
        kn, vn, qn = draw(WIDE, n, hkv, d), draw(WIDE, n, hkv, d), draw(WIDE, n, hq, d)
        q, a, w = (torch.zeros_like(qn) for _ in range(3))
        outs.extend([a, w])
        yield lambda: rkv.rkv_append_rotary(desc, k, v, kn, vn, seq, cap - 1, 1, t, rotary, qn, q)
        if samples:
            yield lambda: rkv.rkv_prefix_attention(desc, k, v, q, seq, a, cap - 1, 1, prefix)
        yield lambda: rkv.rkv_window_attention(desc, k, v, q, seq, w, cap - 1, 1, t, window, 4)

    outs, todo = [], []
    for i, t in enumerate(pieces):
        todo += calls(t, 100 * (i & 1), False)
        for _ in range(3):
            todo += calls(one, 0, True)
    torch.cuda.synchronize()
    for call in todo:
        assert call() == 0
        if wait:
            torch.cuda.synchronize()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return outs + [k, v, seq]


@pytest.mark.parametrize("dtype,d", SHAPES)
@pytest.mark.parametrize("batch", [2, 24])
def test_pieces_of_prompts_and_steps_of_every_type_without_waiting(rkv, dtype, d, batch):
    """Every chain of kernels behind every other one on the same workspace; prefixes read beside the own rows, and apart."""
    want = _mixed_chain(rkv, dtype, d, batch, True)
    for _ in range(3):
        for a, b in zip(_mixed_chain(rkv, dtype, d, batch, False), want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("dtype,d", SHAPES)
@pytest.mark.parametrize("batch,prefixes,rows,cap", [(2, 2, 384, 256), (48, 1, 2048, 384), (200, 1, 4096, 128)])
@pytest.mark.parametrize("paged", [False, True])
def test_captured_calls_of_every_type(rkv, dtype, d, batch, prefixes, rows, cap, paged):
    s = Setup(rkv, dtype, d, 2, 8, [(37 * b) % cap for b in range(batch)], [rows - 5] * prefixes, cap, rows, paged=paged).run()
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
