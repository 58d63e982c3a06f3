"""GPU parity of the paged 8-bit KV cache (Kv8Cache) with its definition in 64 bits (kv8_reference): tables, appended rows, attention,
and a run of them together.  Tables and what the cache holds are compared exactly, attention within the bound that
Kv8Model.tolerance derives."""
import numpy as np
import pytest

from gpu_common import gpu_available
from kv8_reference import PAGE, Kv8Model

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]

HEADS = [(4, 2, 32), (14, 2, 64), (32, 8, 128), (8, 8, 128), (16, 1, 64)]


class Pair:
    """A cache and its model, driven with the same calls."""

    def __init__(self, heads, max_batch, max_seq, n_pages=0, max_rows=None, n_layers=1, dtype="bf16", seed=0):
        import torch
        from paper_2512_15176_amd import Kv8Cache
        self.torch, self.heads, self.dtype = torch, heads, dtype
        self.kv = Kv8Cache(n_layers, *heads, max_batch, max_seq, n_pages=n_pages, max_rows=max_rows)
        self.model = Kv8Model(n_layers, *heads, max_batch, max_seq, n_pages)
        self.rng = np.random.default_rng(seed)

    def dev(self, x, dtype=None):
        t = self.torch.from_numpy(np.ascontiguousarray(x)).cuda()
        return t if dtype is None else t.to(dtype)

    def ints(self, x):
        return self.dev(np.asarray(x, np.int32))

    def rows(self, *shape, scale=1.0):
        """Values that the dtype holds, so that both sides see the same numbers."""
        x = self.dev(scale * self.rng.standard_normal(shape).astype(np.float32))
        t = x.to(self.torch.bfloat16) if self.dtype == "bf16" else x
        return t, t.float().cpu().numpy()

    def reserve(self, start, new, rows=None, max_new=None, max_len=None, check=True):
        rows = sum(new) if rows is None else rows
        max_new = max(new) if max_new is None else max_new
        max_len = max(s + n for s, n in zip(start, new)) if max_len is None else max_len
        slots = self.kv.reserve(self.ints(start), self.ints(new), rows, max_new, max_len)
        want = self.model.reserve(start, new, rows, max_new, max_len)
        if check:
            n = rows
            assert np.array_equal(slots.cpu().numpy(), want[0])
            assert np.array_equal(self.kv.row_seq[:n].cpu().numpy(), want[1]) and np.array_equal(self.kv.row_pos[:n].cpu().numpy(), want[2])
            table = self.kv.block_table.cpu().numpy()
            for b, t in enumerate(self.model.table):
                assert table[b, :len(t)].tolist() == t and (table[b, len(t):] == -1).all(), b
            assert self.kv.lengths.cpu().tolist() == self.model.len
            assert self.kv.status() == (len(self.model.free), want[3])
        return want

    def append(self, layer=0, scale=1.0):
        n, (_, hkv, hd) = self.kv.rows, self.heads
        k, kn = self.rows(n, hkv, hd, scale=scale)
        v, vn = self.rows(n, hkv, hd, scale=scale)
        self.kv.append(layer, k, v)
        self.model.append(layer, kn, vn)

    def read(self, layer=0):
        seq = [b for b, n in enumerate(self.model.len) for _ in range(n)]
        pos = [i for n in self.model.len for i in range(n)]
        if not seq:
            return
        k, v = self.kv.read(layer, self.ints(seq), self.ints(pos), dtype=self.torch.float32)
        want = self.model.read(layer, seq, pos)
        assert np.array_equal(k.cpu().numpy(), want[0], equal_nan=True) and np.array_equal(v.cpu().numpy(), want[1], equal_nan=True)

    def attend(self, layer=0, limits=None, scale=0.0, q_scale=1.0, q=None):
        q, qn = self.rows(self.kv.rows, self.heads[0], self.heads[2], scale=q_scale) if q is None else q
        out = self.kv.attend(layer, q, limits=None if limits is None else self.ints(limits), scale=scale)
        assert out.dtype == q.dtype
        got = out.float().cpu().numpy()
        want = self.model.attend(layer, qn, limits, scale)
        tol = self.model.tolerance(self.dtype, *want)
        nan = np.isnan(want[0])
        assert np.array_equal(nan, np.isnan(got))
        worst = np.abs(got - want[0])[~nan] - tol[~nan]
        assert worst.size == 0 or worst.max() <= 0, (worst.max(), np.abs(got - want[0])[~nan].max())
        return out


# ---------------------------------------------------------------------------------------------------------------- tables
@pytest.mark.parametrize("batch,n_pages,seed", [(1, 0, 1), (5, 20, 2), (64, 300, 3), (1024, 3000, 4)])
def test_tables_over_many_passes(batch, n_pages, seed):
    p = Pair(HEADS[0], batch, 1024, n_pages=n_pages, max_rows=batch * 200, seed=seed)
    rng = p.rng
    for step in range(12):
        start, new = [], []
        for b in range(batch):
            n, lo = p.model.len[b], p.model.hot[b] * PAGE
            kind = rng.integers(0, 11)
            if kind == 10:
                start.append(p.model.base[b])
                new.append(int(min(rng.choice([0, 3, 70]), 1024 - start[-1])))
                continue
            s = n if kind < 5 or n == 0 else 0 if kind == 5 else int(rng.integers(min(lo, n), n + 1)) if kind < 9 else int(rng.integers(0, n + 1)) // PAGE * PAGE
            start.append(s)
            new.append(int(min(rng.choice([0, 1, 33, 64, 65, 200]), 1024 - s)))
        p.reserve(start, new)
    p.kv.close()


def test_tables_refuse_one_by_one():
    p = Pair(HEADS[0], 4, 512, n_pages=6, max_rows=600)
    p.reserve([0, 0, 0, 0], [200, 70, 1, 0])                # 4 + 2 pages: the third sequence does not fit
    assert p.model.len[:3] == [200, 70, 0]
    p.reserve([0, 70, 0, 0], [0, 1, 64, 0])                 # the first gives its pages back and the third takes one of them
    p.reserve([1, 71, 64, -1], [1, 1, 1, 1])                # a start beyond the tokens; a negative one
    p.reserve([0, 72, 65, 0], [1, -3, 500, 0], rows=10, max_new=4, max_len=512)   # numbers out of bounds
    p.reserve([0, 72, 65, 0], [3, 4, 5, 0], rows=10)        # more rows than the bound: the third has no room
    p.reserve([0, 0, 0, 0], [0, 0, 0, 0], rows=0, max_new=0, max_len=0)
    assert p.kv.status() == (6, 0)
    p.kv.close()


def test_a_start_inside_a_page_that_has_cooled_is_refused():
    p = Pair(HEADS[0], 1, 1024, max_rows=1024)
    p.reserve([0], [500])
    assert p.reserve([300], [4])[3] == 1                    # page 4: only 6 and 7 are in the ring
    assert p.reserve([256], [4])[3] == 0                    # a page's start is always possible
    p.append()
    p.read()
    p.kv.close()


def test_the_last_pass_can_be_taken_back():
    """Whole, whatever its length, and a long one again and again, by shorter and longer passes."""
    p = Pair(HEADS[1], 2, 1024, max_rows=1300, seed=6)
    p.reserve([0, 0], [90, 61])
    p.append()
    for start, new in (([90, 61], [500, 300]), ([90, 61], [5, 40]), ([90, 61], [200, 200]), ([70, 61], [300, 299]), ([70, 61], [300, 3]),
                       ([65, 61], [64, 64]), ([66, 62], [0, 0]), ([66, 62], [10, 11])):
        assert p.reserve(start, new)[3] == 0, (start, new)
        p.append()
        p.attend()
        p.read()
    p.reserve([66, 62], [200, 200])
    p.append()
    p.reserve([66, 62], [0, 0])                             # back without rows, and on from there
    p.read()
    p.reserve([66, 62], [70, 70])
    p.append()
    p.attend()
    p.read()
    p.kv.close()


# ---------------------------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS)
def test_what_the_cache_holds(heads, dtype):
    p = Pair(heads, 3, 512, max_rows=600, dtype=dtype, seed=heads[0])
    p.reserve([0, 0, 0], [1, 64, 130])
    p.append()
    p.read()
    p.reserve([1, 64, 130], [33, 1, 200])                   # a long pass that goes on inside a page
    p.append(scale=30.0)
    p.read()
    p.reserve([34, 65, 330], [31, 63, 33])                  # a short one; pages fill
    p.append(scale=1e-3)
    p.read()
    p.reserve([60, 100, 340], [10, 30, 5])                  # rejected rows are written again
    p.append()
    p.read()
    p.kv.close()


def test_rows_of_a_fused_projection_and_extreme_values():
    import torch
    heads = (8, 2, 64)
    p = Pair(heads, 2, 256, max_rows=256)
    p.reserve([0, 0], [128, 70])
    n, (hq, hkv, hd) = 198, heads
    x = p.rng.standard_normal((n, (hq + 2 * hkv) * hd)).astype(np.float32)
    x[:64, hq * hd] = 448.0                                  # a page whose largest value is exactly 448, and one just above it
    x[64:128, hq * hd + 1] = 450.0
    x[0, (hq + hkv) * hd:] = 0.0
    x[64:128, (hq + hkv) * hd:] = 0.0                        # a page of zeros
    x[128:, hq * hd:] *= 1e30                                # large and small magnitudes
    x[140:, (hq + hkv) * hd:] = 1e-35
    t = p.dev(x).to(torch.bfloat16)
    k, v = t[:, hq * hd:(hq + hkv) * hd].unflatten(1, (hkv, hd)), t[:, (hq + hkv) * hd:].unflatten(1, (hkv, hd))
    p.kv.append(0, k, v)
    p.model.append(0, k.float().cpu().numpy(), v.float().cpu().numpy())
    p.read()
    p.kv.close()


# ---------------------------------------------------------------------------------------------------------------- attention
PASSES = [   # tokens before the pass, rows
    ([0], [1]), ([63], [1]), ([64], [1]), ([700], [1]), ([0], [64]), ([0], [65]), ([100], [32]), ([0], [333]), ([190], [150]),
    ([0, 5, 64, 700, 1, 127, 900], [7, 1, 33, 0, 64, 2, 31]), ([900, 10], [1, 1]),
]


@pytest.mark.parametrize("heads,dtype", [(h, "bf16") for h in HEADS] + [(h, "f32") for h in HEADS[:3]])
@pytest.mark.parametrize("start,new", PASSES)
def test_attention(heads, dtype, start, new):
    p = Pair(heads, len(start), 1024, max_rows=max(sum(start) + 1, sum(new)), dtype=dtype, seed=sum(start) + sum(new))
    if max(start):
        p.reserve([0] * len(start), start)
        p.append()
    p.reserve(start, new)
    p.append()
    p.attend(q_scale=2.0)
    end = [s + n for s, n in zip(start, new)]
    every = [e for e, n in zip(end, new) for _ in range(n)]
    p.attend(limits=every)                                   # all see all
    p.attend(limits=[int(p.rng.integers(-2, e + 3)) for e in every], scale=0.3)   # any number of keys, none among them
    p.attend(limits=[0] * len(every))
    p.attend(limits=[0 if i % 3 == 1 else e for i, e in enumerate(every)])      # rows that see nothing among rows that see all
    p.kv.close()


@pytest.mark.parametrize("heads", HEADS[:3])
def test_rows_one_by_one_are_the_block(heads):
    """A block of rows, the same rows one at a time, and the same tokens as a prompt: what a row reads goes by its position."""
    import torch
    hq, hkv, hd = heads
    n0, n = 120, 20
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v, q = (torch.randn(n0 + n, h, hd, generator=g, device="cuda") for h in (hkv, hkv, hq))
    from paper_2512_15176_amd import Kv8Cache
    outs = []
    for pieces in ([n0, n], [n0] + [1] * n, [n0 + n]):
        kv = Kv8Cache(1, hq, hkv, hd, 1, 256, max_rows=256)
        at, got = 0, []
        for m in pieces:
            one = torch.tensor([at], dtype=torch.int32, device="cuda")
            kv.reserve(one, torch.full_like(one, m), m, m, at + m)
            kv.append(0, k[at:at + m], v[at:at + m])
            got.append(kv.attend(0, q[at:at + m]))
            at += m
        outs.append(torch.cat(got)[n0:])
        kv.close()
    # float32 throughout: the same keys, summed in other orders
    for o in outs[1:]:
        assert (o - outs[0]).abs().max() < 2e-5


def test_rejected_drafts_leave_no_trace():
    p = Pair(HEADS[1], 2, 512, max_rows=256, seed=9)
    p.reserve([0, 0], [60, 101])
    p.append()
    for start, scale in (([60, 101], 100.0), ([61, 130], 1.0), ([70, 127], 50.0), ([66, 140], 1.0)):   # pages fill and are taken back
        p.reserve(start, [32, 30])
        p.append(scale=scale)
        p.attend()
        p.read()
    p.kv.close()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("where", ["k", "v"])
def test_infinities_and_nans_reach_only_the_rows_that_see_them(bad, where):
    import torch
    heads = (8, 2, 64)
    p = Pair(heads, 2, 256, max_rows=256, seed=3)
    p.reserve([0, 0], [100, 70])
    kn = p.rng.standard_normal((170, 2, 64)).astype(np.float32)
    vn = p.rng.standard_normal((170, 2, 64)).astype(np.float32)
    (kn if where == "k" else vn)[90, 1, 7] = bad             # token 90 of the first sequence, second kv head
    k, v = p.dev(kn).to(torch.bfloat16), p.dev(vn).to(torch.bfloat16)
    p.kv.append(0, k, v)
    p.model.append(0, k.float().cpu().numpy(), v.float().cpu().numpy())
    out = p.attend()
    assert torch.isnan(out[90:100, 4:]).all() and not torch.isnan(out[:90]).any() and not torch.isnan(out[:, :4]).any() and not torch.isnan(out[100:]).any()
    p.reserve([100, 70], [40, 0])                            # the page fills: the same from 8 bits
    p.append()
    p.attend(limits=[90] * 20 + [91] * 20)
    p.reserve([90, 70], [2, 3])                              # and it is taken back
    p.append()
    assert not torch.isnan(p.attend()).any()
    p.kv.close()


def test_refused_rows_come_out_as_zeros():
    p = Pair(HEADS[2], 3, 256, n_pages=2, max_rows=256)
    assert p.reserve([0, 0, 0], [40, 90, 60])[3] == 2
    p.append()
    out = p.attend()
    assert (out[40:] == 0).all() and (out[:40] != 0).any()
    p.kv.close()


def test_rows_behind_the_pass_are_left_alone():
    import torch
    p = Pair(HEADS[2], 2, 256, max_rows=256)
    p.reserve([0, 0], [5, 3], rows=12)                       # the bound is larger than the sum
    hq, hkv, hd = HEADS[2]
    k, v, q = (torch.randn(12, h, hd, device="cuda", dtype=torch.bfloat16) for h in (hkv, hkv, hq))
    p.kv.append(0, k, v)
    p.model.append(0, k.float().cpu().numpy(), v.float().cpu().numpy())
    out = torch.full((14, hq + 1, hd), 7.0, device="cuda", dtype=torch.bfloat16)
    view = out[1:13, :hq]                                    # strided rows
    p.kv.attend(0, q, out=view)
    want = p.model.attend(0, q.float().cpu().numpy())
    tol = p.model.tolerance("bf16", *want)
    assert (np.abs(view[:8].float().cpu().numpy() - want[0][:8]) <= tol[:8]).all()
    assert (out[9:] == 7).all() and (out[0] == 7).all() and (out[:, hq] == 7).all()
    p.kv.close()


def test_long_contexts_and_key_ranges():
    """Contexts of which a workgroup takes a share, for one row, a block of a group and a block of single heads."""
    for heads, start, new in (((8, 2, 128), [9000, 100], [1, 1]), ((8, 2, 128), [9000, 64], [31, 17]), ((4, 4, 64), [9000, 3000], [3, 40])):
        p = Pair(heads, 2, 9216, max_rows=sum(start), seed=start[1])
        p.reserve([0, 0], start)
        p.append()
        p.reserve(start, new)
        p.append()
        p.attend(q_scale=3.0)
        p.kv.close()


def test_a_pool_of_more_than_four_gigabytes():
    import torch
    from paper_2512_15176_amd import Kv8Cache
    heads, full = (8, 8, 128), 1 << 20
    kv = Kv8Cache(1, *heads, 3, full, n_pages=33000, max_rows=512)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    # two sequences take the first 32768 pages (4.3 GB), whose rows are never written
    new = [ints([512, 0, 0]), ints([0, 512, 0])]
    for b in range(2):
        for n in range(0, full, 512):
            kv.reserve(ints([full, n, 0] if b else [n, 0, 0]), new[b], 512, 512, full)
    assert kv.status() == (33000 - 32768, 0)
    k, v, q = (torch.randn(200, 8, 128, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    slots = kv.reserve(ints([full, full, 0]), ints([0, 0, 200]), 200, 200, full)
    assert (slots.cpu().numpy() == 32768 * PAGE + np.arange(200)).all()
    kv.append(0, k, v)
    out = kv.attend(0, q)
    small = Pair(heads, 1, 256, max_rows=256)
    small.reserve([0], [200])
    small.kv.append(0, k, v)
    small.model.append(0, k.float().cpu().numpy(), v.float().cpu().numpy())
    want = small.attend(q=(q, q.float().cpu().numpy()))
    assert (out.float() - want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()
    kv.close()
    small.kv.close()


# ---------------------------------------------------------------------------------------------------------------- together
def test_a_decoding_loop_over_two_layers():
    p = Pair((14, 2, 64), 3, 512, n_pages=20, max_rows=400, n_layers=2, dtype="f32", seed=11)
    p.reserve([0, 0, 0], [150, 64, 9])
    for layer in range(2):
        p.append(layer)
        p.attend(layer)
    for step in range(6):
        accepted = [int(x) for x in p.rng.integers(1, 17, 3)]
        start = [n - 16 + a if step else n for n, a in zip(p.model.len, accepted)]
        p.reserve(start, [16, 16, 16])
        for layer in range(2):
            p.append(layer)
            p.attend(layer)
    p.reserve([0, p.model.len[1], 0], [77, 1, 0])            # one sequence ends, another prompt takes its place, one leaves
    for layer in range(2):
        p.append(layer)
        p.attend(layer)
        p.read(layer)
    p.kv.close()


def test_captured_passes_replay():
    """Two captured decoding passes that share a cache, replayed in turn with eager passes between them."""
    import torch
    from paper_2512_15176_amd import Kv8Cache
    hq, hkv, hd = 8, 2, 128
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        caches = [Kv8Cache(1, hq, hkv, hd, 2, 512, max_rows=256) for _ in range(2)]
        start = torch.zeros(2, dtype=torch.int32, device="cuda")
        new = torch.full((2,), 8, dtype=torch.int32, device="cuda")
        k, v, q = (torch.randn(16, h, hd, device="cuda", dtype=torch.bfloat16) for h in (hkv, hkv, hq))

        def one(kv, rows):
            kv.reserve(start, new[:2], rows, 8, 512)
            kv.append(0, k, v)
            return kv.attend(0, q)

        one(caches[0], 16)
        one(caches[0], 16)
        side.synchronize()
        graphs, outs = [], []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                outs.append(one(caches[0], 16))
            graphs.append(g)
        rng = np.random.default_rng(0)
        n = 0
        start.fill_(0)
        caches[0].reserve(start, start, 0, 0, 0)
        caches[1].reserve(start, start, 0, 0, 0)
        for step in range(20):
            start.fill_(n)
            for t, h in ((k, hkv), (v, hkv), (q, hq)):
                t.copy_(torch.from_numpy(rng.standard_normal((16, h, hd)).astype(np.float32)))
            want = one(caches[1], 16).clone()
            if step % 3 == 2:
                got = one(caches[0], 16)
            else:
                graphs[step % 3].replay()
                got = outs[step % 3]
            assert torch.equal(got, want), step
            n += int(rng.integers(1, 9))
        for kv in caches:
            kv.close()


def test_calls_from_another_stream_wait():
    import torch
    p = Pair((8, 2, 128), 1, 4096, max_rows=4096, seed=2)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(10):
            big = big @ big * 1e-3                            # the rows come late
        k = torch.randn(1000, 2, 128, device="cuda", dtype=torch.bfloat16) + 0 * big[:1000, :1, None].nan_to_num(0, 0, 0).to(torch.bfloat16)
        p.reserve([0], [1000])
        p.kv.append(0, k, k)
        out = p.kv.attend(0, k.repeat_interleave(4, 1))
        kn = k.float().cpu().numpy()
    p.model.append(0, kn, kn)
    want = p.model.attend(0, np.repeat(kn, 4, 1))
    assert (np.abs(out.float().cpu().numpy() - want[0]) <= p.model.tolerance("bf16", *want)).all()
    p.kv.close()


def test_arguments_are_checked():
    import torch
    from paper_2512_15176_amd import DeerError, Kv8Cache
    with pytest.raises(DeerError):
        Kv8Cache(1, 6, 4, 64, 1, 64)                         # query heads no multiple of kv heads
    p = Pair((8, 2, 64), 2, 128, max_rows=64)
    x = lambda *s, **kw: torch.zeros(*s, device="cuda", **{"dtype": torch.bfloat16, **kw})   # noqa: E731
    with pytest.raises(DeerError) as e:                      # no tables yet
        p.kv.append(0, x(0, 2, 64), x(0, 2, 64))
    assert e.value.status == -2
    for bad in (dict(rows=65), dict(max_new=129), dict(max_len=129)):
        with pytest.raises(DeerError):
            p.reserve([0, 0], [4, 4], check=False, **{**dict(rows=8), **bad})
    p.reserve([0, 0], [4, 4])
    with pytest.raises(DeerError):
        p.kv.append(1, x(8, 2, 64), x(8, 2, 64))             # no such layer
    for k in (x(7, 2, 64), x(8, 2, 32), x(8, 64, 2).transpose(1, 2), torch.zeros(8, 2, 64)):
        with pytest.raises(ValueError):
            p.kv.append(0, k, k)
    with pytest.raises(TypeError):
        p.kv.append(0, x(8, 2, 64, dtype=torch.float16), x(8, 2, 64, dtype=torch.float16))
    with pytest.raises(DeerError):
        odd = x(8 * 129 + 8)[4:4 + 8 * 129].view(8, 129)[:, :128].unflatten(1, (2, 64))
        p.kv.append(0, odd, odd)                             # neither address nor stride keeps 16 bytes
    with pytest.raises(DeerError):
        p.kv.attend(0, x(8, 8, 64), scale=-1.0)
    with pytest.raises(ValueError):
        p.kv.attend(0, x(8, 8, 64), limits=torch.zeros(8, device="cuda"))
    with pytest.raises(TypeError):
        p.kv.attend(0, x(8, 8, 64), out=x(8, 8, 64, dtype=torch.float32))
    p.append()
    p.attend()
    p.kv.close()
    with pytest.raises(RuntimeError):
        p.kv.attend(0, x(8, 8, 64))


def test_a_captured_loop_over_the_handles_own_lengths():
    """A prompt and single tokens behind what the sequences hold (start: the cache's lengths), captured and replayed over two layers."""
    import torch
    from paper_2512_15176_amd import Kv8Cache
    hq, hkv, hd, L = 8, 2, 64, 2
    rng = np.random.default_rng(17)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a, b = (Kv8Cache(L, hq, hkv, hd, 3, 1024, max_rows=600) for _ in range(2))
        zero = torch.zeros(3, dtype=torch.int32, device="cuda")
        count = {n: torch.tensor([n, 0, n], dtype=torch.int32, device="cuda") for n in (1, 150)}
        data = {n: [torch.randn(2 * n, h, hd, device="cuda", dtype=torch.bfloat16) for h in (hkv, hkv, hq)] for n in (1, 150)}

        def one(kv, start, n):
            kv.reserve(start, count[n], 2 * n, n, 1024)
            outs = []
            for layer in range(L):
                kv.append(layer, data[n][0] * (layer + 1), data[n][1])
                outs.append(kv.attend(layer, data[n][2]))
            return torch.stack(outs)

        for n in (1, 150):
            one(a, a.lengths, n)
        side.synchronize()
        graphs = {}
        for n in (1, 150):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                out = one(a, a.lengths, n)
            graphs[n] = (g, out)
        a.reserve(zero, zero, 0, 0, 0)
        held = [0, 0, 0]
        for n in (150, 1, 1, 150, 1, 150, 1, 1):
            for t in data[n]:
                t.copy_(torch.from_numpy(rng.standard_normal(tuple(t.shape)).astype(np.float32)))
            graphs[n][0].replay()
            want = one(b, torch.tensor(held, dtype=torch.int32, device="cuda"), n)
            held = [held[0] + n, 0, held[2] + n]
            assert torch.equal(graphs[n][1], want) and a.lengths.tolist() == held == b.lengths.tolist()
            taken = a.block_table[a.block_table >= 0].tolist()        # (not b's pages: those that a's first passes gave back lie in another order)
            assert len(taken) == len(set(taken)) == int(a.pages_held.sum()) == sum(-(-x // 64) for x in held)
    a.close()
    b.close()


def test_two_caches_work_at_once():
    """Two handles on two streams, whose passes overlap, give what each gives alone."""
    import torch
    from paper_2512_15176_amd import Kv8Cache
    hq, hkv, hd = 8, 2, 128
    streams = [torch.cuda.Stream() for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v, q = (torch.randn(2, 2000, h, hd, generator=g, device="cuda", dtype=torch.bfloat16) for h in (hkv, hkv, hq))
    n = torch.tensor([2000], dtype=torch.int32, device="cuda")
    zero, one = torch.zeros_like(n), torch.ones_like(n)
    torch.cuda.synchronize()
    outs = {}
    for alone in (True, False):
        caches = []
        for s in streams:
            with torch.cuda.stream(s):
                caches.append(Kv8Cache(1, hq, hkv, hd, 1, 4096, max_rows=2000))
        got = [[], []]
        for i in range(6):
            for j, s in enumerate(streams):
                with torch.cuda.stream(s):
                    if i == 0:
                        caches[j].reserve(zero, n, 2000, 2000, 2000)
                        caches[j].append(0, k[j], v[j])
                        got[j].append(caches[j].attend(0, q[j]))
                    else:
                        caches[j].reserve(caches[j].lengths, one, 1, 1, 4096)
                        caches[j].append(0, k[j, i:i + 1], v[j, i:i + 1])
                        got[j].append(caches[j].attend(0, q[j, i:i + 1]))
                if alone:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        outs[alone] = [torch.cat(x) for x in got]
        for kv in caches:
            kv.close()
    for j in range(2):
        assert torch.equal(outs[True][j], outs[False][j])


@pytest.mark.parametrize("heads,dtype", [((3, 3, 32), "bf16"), ((10, 2, 64), "f32"), ((64, 1, 128), "bf16"), ((192, 3, 32), "f32"), ((6, 1, 128), "f32")])
def test_groups_that_fill_no_tile_and_groups_of_64(heads, dtype):
    p = Pair(heads, 5, 512, max_rows=1200, dtype=dtype, seed=heads[0])
    start = [0, 31, 130, 300, 64]
    p.reserve([0] * 5, start)
    p.append()
    p.reserve(start, [1, 5, 33, 0, 2])
    p.append()
    p.attend()
    p.reserve([130, 31, 0, 300, 66], [3, 0, 0, 70, 0], check=False)      # the first has too few tokens, the third leaves
    p.append()
    p.attend(scale=0.1)
    p.kv.close()


def test_a_thousand_sequences_and_ranges_of_keys_in_part_of_the_chip():
    p = Pair((4, 2, 32), 1024, 128, n_pages=1500, max_rows=4096, seed=6)
    start = [int(x) for x in p.rng.integers(0, 6, 1024)]
    p.reserve([0] * 1024, start)
    p.append()
    p.reserve(start, [(b * 7) % 3 for b in range(1024)])
    p.append()
    p.attend()
    p.kv.close()
    for heads, dtype, batch, new in (((32, 8, 128), "bf16", 14, 12), ((14, 2, 64), "f32", 16, 21), ((32, 8, 128), "bf16", 3, 32)):
        p = Pair(heads, batch, 2048, max_rows=20000, dtype=dtype, seed=batch)
        start = [900 + 25 * b for b in range(batch)]
        p.reserve([0] * batch, start)
        p.append()
        p.reserve(start, [new - b % 2 for b in range(batch)])
        p.append()
        p.attend(q_scale=2.0)
        p.kv.close()


@pytest.mark.parametrize("batch", [2, 127, 128, 129])
def test_sequences_of_equal_and_unequal_lengths_in_any_order(batch):
    p = Pair((14, 2, 64), batch, 512, max_rows=40 * batch if batch > 2 else 1000, seed=batch)
    start = [int(x) for x in p.rng.choice([0, 1, 7, 7, 35], batch)] if batch > 2 else [30, 330]
    p.reserve([0] * batch, start)
    p.append()
    p.reserve(start, [int(x) for x in p.rng.choice([0, 1, 3, 3], batch)] if batch > 2 else [150, 150])
    p.append()
    p.attend()
    p.kv.close()
