"""rkv_append_rotary on the GPU against the plain form in 64 bits."""
import pytest
import torch

from tokens_util import TYPES, WIDE, descriptor, from_pages, random_rows, rotate, rotation_table, rounding_tolerance, to_pages

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rkv():
    from paper_2505_24133_b200 import build as b
    b.build()
    import paper_2505_24133_b200 as r
    assert r.lib() is not None
    return r


def _bytes(t):
    return t.contiguous().view(torch.uint8)


class Setup:
    def __init__(self, rkv, dtype, d, hkv, hq, lens, new, cap, seed, rotary=None, interleaved=False, paged=False, rows=4096, fused=False,
                 positions=None, behind=0, longest=None, offsets=True):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        B, total = len(lens), sum(new) + behind
        self.rkv, self.dtype, self.d, self.hkv, self.hq, self.cap = rkv, dtype, d, hkv, hq, cap
        self.lens0, self.new = list(lens), list(new)
        self.k, self.v = (random_rows((B, hkv, cap, d), dtype, gen) for _ in range(2))
        self.table = None
        if paged:
            self.pool_k, self.table = to_pages(self.k, gen)
            flat = self.table.flatten().long()
            self.pool_v = torch.zeros_like(self.pool_k)
            _bytes(self.pool_v)[flat] = _bytes(self.v).view(flat.numel(), 128, -1)
        wide = WIDE[dtype]
        qkv = torch.randn(total, hq + 2 * hkv, d, generator=gen, device="cuda").to(wide)
        parts = [qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]]
        self.q_new, self.k_new, self.v_new = parts if fused else [x.contiguous() for x in parts]
        self.q_out = torch.full((total, hq, d), 7.0, device="cuda", dtype=wide)
        self.seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.dim = d if rotary is None else rotary
        self.interleaved = interleaved
        self.angles = rotation_table(rows, self.dim) if self.dim else None
        self.pos = [5 * b for b in range(B)] if positions is None else positions
        self.positions = torch.tensor(self.pos, dtype=torch.int32, device="cuda")
        off = [sum(new[:b]) for b in range(B + 1)]
        self.offsets = torch.tensor(off, dtype=torch.int32, device="cuda") if offsets else None
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        stride = dict(q_stride=qkv.stride(0), k_stride=qkv.stride(0), v_stride=qkv.stride(0)) if fused else {}
        self.tokens = rkv.rkv_tokens(total, longest or max(max(new), 1), self.offsets, **stride)
        self.rotary = rkv.rkv_rotary(self.angles, self.dim, self.positions, interleaved)
        self.desc = descriptor(rkv, B, hkv, hq, d, dtype, self.status, self.table, self.pool_k.shape[0] if paged else 0)

    def caches(self):
        return (self.pool_k, self.pool_v) if self.table is not None else (self.k, self.v)

    def call(self, q=True, stream=None, q_out=None):
        k, v = self.caches()
        return self.rkv.rkv_append_rotary(self.desc, k, v, self.k_new, self.v_new, self.seq, self.cap - 1, 1, self.tokens, self.rotary,
                                          self.q_new if q else None, (self.q_out if q_out is None else q_out) if q else None, stream)

    def check(self, refused=(), q=True):
        """Everything the call has to have written, and everything else as it was before."""
        want_k, want_v = self.k.clone(), self.v.clone()
        k, v = self.after
        first = 0
        q_seen = torch.zeros(self.q_out.shape[0], dtype=torch.bool, device="cuda")
        for b, n in enumerate(self.new):
            rows = slice(self.lens0[b], self.lens0[b] + n)
            if b not in refused and n:
                t = slice(first, first + n)
                pos = self.pos[b] + torch.arange(n, device="cuda")
                for name, src, cache, want in (("k", self.k_new, k, want_k), ("v", self.v_new, v, want_v)):
                    ref, size = rotate(src[t].double(), pos, self.dim if name == "k" else 0, self.interleaved)
                    got = cache[b, :, rows].transpose(0, 1)
                    if name == "v" and self.dtype != "fp8":
                        assert torch.equal(_bytes(got), _bytes(src[t]))
                    tol = rounding_tolerance(ref, size, TYPES[self.dtype])
                    over = float(((got.double() - ref).abs() - tol).max())
                    assert over <= 0, (name, b, over)
                    _bytes(want)[b, :, rows] = _bytes(cache)[b, :, rows]
                if q:
                    ref, size = rotate(self.q_new[t].double(), pos, self.dim, self.interleaved)
                    over = float(((self.q_out[t].double() - ref).abs() - rounding_tolerance(ref, size, WIDE[self.dtype])).max())
                    assert over <= 0, ("q", b, over)
                    q_seen[t] = True
            first += n
        assert torch.equal(_bytes(k), _bytes(want_k)) and torch.equal(_bytes(v), _bytes(want_v))     # nothing else is touched
        assert (self.q_out[~q_seen] == 7.0).all()
        assert self.seq.tolist() == [L + (0 if b in refused else n) for b, (L, n) in enumerate(zip(self.lens0, self.new))]
        assert int(self.status.item()) == (1 if refused else 0)

    def run(self, refused=(), **kw):
        before = self.k.clone(), self.v.clone()
        assert self.call(**kw) == 0
        torch.cuda.synchronize()
        if self.table is None:
            self.after = self.k, self.v
            self.k, self.v = before
        else:
            self.after = from_pages(self.pool_k, self.table, self.d), from_pages(self.pool_v, self.table, self.d)
        self.check(refused, q=kw.get("q", True))


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("d,rotary,interleaved", [(128, 128, False), (128, 64, True), (64, 64, True), (64, 16, False), (256, 256, False),
                                                  (256, 128, True), (128, 0, False)])
def test_one_token_per_sequence(rkv, dtype, d, rotary, interleaved):
    """An empty cache, one with a single free row, lengths in between; the last cache is full, and one position has no table row."""
    lens = [0, 99, 17, 100, 50]
    s = Setup(rkv, dtype, d, 2, 6, lens, [1] * 5, 100, 11, rotary, interleaved, positions=[0, 4095, 700, 3, 4096], offsets=False)
    s.run(refused=(3, 4) if rotary else (3,))


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("d,rotary,interleaved,paged,fused", [(128, 128, False, True, True), (128, 96, True, False, True),
                                                              (64, 64, False, True, False), (256, 64, True, True, True), (128, 0, False, True, True)])
def test_ragged_prompts(rkv, dtype, d, rotary, interleaved, paged, fused):
    """Sequences without tokens first, last and in between, one that fills its cache, one that is a row too long, rows behind the last."""
    lens = [0, 3, 0, 130, 250, 100, 256, 7]
    new = [0, 5, 131, 1, 6, 157, 0, 0]
    s = Setup(rkv, dtype, d, 3, 6, lens, new, 256, 12, rotary, interleaved, paged, fused=fused, behind=4)
    s.run(refused=(5,))


@pytest.mark.parametrize("batch,new", [(1, 3), (1, 700), (33, 2), (70, 9), (1100, 3)])
@pytest.mark.parametrize("offsets", [False, True])
def test_sequences_are_found(rkv, batch, new, offsets):
    """Batches below, at and beyond what one look at 32 offsets finds, with and without offsets."""
    s = Setup(rkv, "bf16", 64, 1, 2, [b % 5 for b in range(batch)], [new] * batch, new + 8, 13, offsets=offsets, rows=8192)
    s.run()


@pytest.mark.parametrize("hkv,hq", [(1, 1), (1, 16), (16, 16), (40, 160)])
@pytest.mark.parametrize("step", [True, False])
def test_head_layouts(rkv, hkv, hq, step):
    s = Setup(rkv, "bf16", 128, hkv, hq, [4, 0, 9], [1, 1, 1] if step else [3, 1, 2], 16, 14, offsets=not step)
    s.run()


def test_without_queries_and_rotated_in_place(rkv):
    s = Setup(rkv, "bf16", 128, 2, 4, [1, 2], [4, 9], 64, 15)
    s.run(q=False)
    s = Setup(rkv, "bf16", 128, 2, 4, [1, 2], [4, 9], 64, 15)
    other = Setup(rkv, "bf16", 128, 2, 4, [1, 2], [4, 9], 64, 15)
    assert s.call() == 0
    assert other.call(q_out=other.q_new) == 0
    torch.cuda.synchronize()
    assert torch.equal(s.q_out, other.q_new)


def test_positions_default_to_the_rows(rkv):
    s = Setup(rkv, "bf16", 128, 1, 2, [3, 40], [4, 9], 64, 16, positions=[3, 40])
    s.rotary = rkv.rkv_rotary(s.angles, 128)
    s.run()


def test_bad_lengths_positions_and_offsets_are_refused_one_by_one(rkv):
    s = Setup(rkv, "bf16", 128, 2, 4, [10, -1, 65, 20, 30], [4] * 5, 64, 17, positions=[0, 0, 0, -1, 4093])
    s.run(refused=(1, 2, 3, 4))
    s = Setup(rkv, "bf16", 128, 2, 4, [10, 5, 6], [4, 4, 4], 64, 18)          # one has more tokens than the call said
    s.offsets.copy_(torch.tensor([0, 4, 11, 12], dtype=torch.int32))
    s.tokens.longest, s.new = 4, [4, 7, 1]
    s.run(refused=(1,))
    s = Setup(rkv, "bf16", 128, 2, 4, [10, 5], [4, 4], 64, 19)                # one ends behind the tensors
    s.offsets.copy_(torch.tensor([0, 4, 9], dtype=torch.int32))
    s.tokens.longest = 9
    s.run(refused=(1,))


def test_pages_that_do_not_exist_are_not_written(rkv):
    s = Setup(rkv, "bf16", 64, 2, 2, [100, 100], [60, 60], 256, 20, paged=True)
    s.table[0, 1, 1], s.table[1, 0, 0] = -1, s.pool_k.shape[0]
    before = s.pool_k.clone()
    good = s.table.clone()
    assert s.call() == 0
    torch.cuda.synchronize()
    assert int(s.status.item()) == 1
    named = torch.zeros(s.pool_k.shape[0], dtype=torch.bool, device="cuda")
    named[good[(good >= 0) & (good < s.pool_k.shape[0])].long()] = True
    assert torch.equal(_bytes(s.pool_k)[~named], _bytes(before)[~named])
    assert not torch.equal(_bytes(s.pool_k)[named], _bytes(before)[named])


def test_rounding_to_codes_saturates_and_keeps_nan(rkv):
    s = Setup(rkv, "fp8", 64, 1, 1, [0], [2], 4, 21, rotary=0)
    s.v_new[0, 0, :6] = torch.tensor([1e9, -1e9, 448.0, float("inf"), -float("inf"), float("nan")], dtype=torch.bfloat16)
    assert s.call() == 0
    torch.cuda.synchronize()
    got = s.v[0, 0, 0, :6].float().tolist()
    assert got[:5] == [448.0, -448.0, 448.0, 448.0, -448.0] and got[5] != got[5]


def test_rows_beyond_32_bits(rkv):
    """A cache of more than 2^31 elements: its last head's last rows."""
    hkv, cap, d = 20, 1 << 20, 128
    k = torch.zeros(1, hkv, cap, d, dtype=torch.float8_e4m3fn, device="cuda")
    v = torch.zeros_like(k)
    seq = torch.tensor([cap - 3], dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(22)
    new = torch.randn(3, hkv, d, generator=gen, device="cuda").to(torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = descriptor(rkv, 1, hkv, hkv, d, "fp8", status)
    assert rkv.rkv_append_rotary(desc, k, v, new, new, seq, cap - 1, 1, rkv.rkv_tokens(3, 3), rkv.rkv_rotary(None, 0)) == 0
    torch.cuda.synchronize()
    want = new.transpose(0, 1).float().to(torch.float8_e4m3fn)
    assert torch.equal(_bytes(k[0, :, cap - 3:]), _bytes(want)) and torch.equal(_bytes(v[0, :, cap - 3:]), _bytes(want))
    assert int(seq.item()) == cap and int(status.item()) == 0
    assert int((_bytes(k) != 0).sum()) == int((_bytes(want) != 0).sum())


def test_another_stream_and_a_captured_graph(rkv):
    """Two steps and a prompt in one graph, replayed on restored caches, against the same calls made eagerly on a stream of their own."""
    s = Setup(rkv, "bf16", 128, 2, 4, [3, 9], [1, 1], 64, 23, offsets=False)
    p = Setup(rkv, "bf16", 128, 2, 4, [5, 11], [6, 2], 64, 24)
    p.k, p.v, p.seq = s.k, s.v, s.seq
    k0, v0, l0 = s.k.clone(), s.v.clone(), s.seq.clone()

    def steps(stream=None):
        assert s.call(stream=stream) == 0 and s.call(stream=stream) == 0 and p.call(stream=stream) == 0

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    steps(side)
    torch.cuda.synchronize()
    want = s.k.clone(), s.v.clone(), s.seq.clone(), p.q_out.clone()
    assert s.seq.tolist() == [11, 13]

    def restore():
        s.k.copy_(k0), s.v.copy_(v0), s.seq.copy_(l0), p.q_out.zero_()

    restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        steps()
    for _ in range(2):
        restore()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s.k, want[0]) and torch.equal(s.v, want[1]) and torch.equal(s.seq, want[2]) and torch.equal(p.q_out, want[3])
