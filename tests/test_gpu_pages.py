"""GPU parity of the page calls (reserve, fork, free, copy, compact) with a plain model of the table, the counts and the pools: all equal to
the bit, also where requests are refused."""
import numpy as np
import pytest
import torch

from paper_2603_08899_b200 import binding as cb
from tests import harness as H
from tests.block_ref import PAGE, to_cuda

pytestmark = pytest.mark.gpu


class Model:
    """Table, counts and, of each layer, a number per page that stands for its contents."""

    def __init__(self, n_pages, n_rows, max_pages, seed, kind="bf16", L=2, Hkv=2, D=64, block=32):
        self.r = np.random.RandomState(seed)
        self.n_pages, self.table, self.ref = n_pages, np.full((n_rows, max_pages), -1, np.int32), np.zeros(n_pages, np.int32)
        self.kind, self.L, self.block = kind, L, block
        dt = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.uint8, "block": torch.uint8}[kind]
        self.dims = cb.make_dims(1, Hkv, Hkv, D, 1, 0, 0, cb.FP8_BLOCK if kind == "block" else dt)
        shape = (n_pages * PAGE, Hkv, D)
        self.regs = []
        self.pools = []
        for _ in range(2 * L):
            t = H.guarded(self.regs, shape, dt)
            t.view(torch.int16 if dt != torch.float32 else torch.int32).random_()
            self.pools.append(t)
        self.scales = []
        for _ in range(2 * L if kind == "block" else 0):
            t = H.guarded(self.regs, (n_pages, Hkv, PAGE // block), torch.float32)
            t.uniform_()
            self.scales.append(t)
        self.want = [t.clone() for t in self.pools + self.scales]
        self.d_table, self.d_ref = to_cuda(self.table), to_cuda(self.ref)
        self.ctx = cb.confu_create(0)
        ptr = lambda ts: torch.tensor([t.data_ptr() for t in ts], dtype=torch.int64, device="cuda")  # noqa: E731
        self.k, self.v = ptr(self.pools[:L]), ptr(self.pools[L:])
        if kind == "block":
            self.ks, self.vs = ptr(self.scales[:L]), ptr(self.scales[L:])
            cb.confu_set_kv_block_scale_layers(self.ctx, self.ks, self.vs, block)
        self.pages = cb.make_pages(self.d_ref, self.d_table)
        self.ws = H.guarded(self.regs, (cb.confu_pages_workspace_bytes(n_pages),), torch.uint8)

    def close(self):
        cb.confu_destroy(self.ctx)

    def status(self, n):
        self.d_status = H.guarded(self.regs, (max(n, 1),), torch.int32, 0)
        return self.d_status[:n]

    def copy_pages(self, pairs):
        for t in self.want:
            pages = t.view(self.n_pages, -1)
            for s, d in pairs:
                pages[d] = pages[s]

    def check(self, status=None, codes=None, what=""):
        torch.cuda.synchronize()
        assert np.array_equal(self.d_table.cpu().numpy(), self.table), what
        assert np.array_equal(self.d_ref.cpu().numpy(), self.ref), what
        for got, want in zip(self.pools + self.scales, self.want):
            assert torch.equal(got.view(torch.uint8), want.view(torch.uint8)), what
        if status is not None:
            assert status.tolist() == codes, what
        H.assert_guards(self.regs, what or "page calls")
        # the counts are what the table says
        named = self.table[self.table >= 0]
        assert np.array_equal(np.bincount(named, minlength=self.n_pages), self.ref), what

    def free_pages(self):
        return [p for p in range(self.n_pages) if self.ref[p] == 0]

    # ---- the calls, on both sides
    def reserve(self, rows, lengths, stream=None):
        st = self.status(len(rows))
        cb.confu_pages_reserve(self.ctx, self.pages, to_cuda(np.array(rows, np.int32)), to_cuda(np.array(lengths, np.int32)), st, stream)
        codes, free, out, seen = [], self.free_pages(), False, []
        for row, n in zip(rows, lengths):
            need = -(-n // PAGE)
            code = 0
            if not 0 <= row < len(self.table) or n < 0 or need > self.table.shape[1] or row in seen:
                code = cb.ST_BAD_PAGES
            else:
                lacks = [j for j in range(need) if self.table[row, j] < 0]
                if lacks and (out or len(lacks) > len(free)):
                    code, out = cb.ST_NO_PAGES, True
                else:
                    for j in lacks:
                        self.table[row, j] = free.pop(0)
                        self.ref[self.table[row, j]] = 1
            seen.append(row)
            codes.append(code)
        self.check(st, codes, "reserve")

    def free(self, rows):
        st = self.status(len(rows))
        cb.confu_pages_free(self.ctx, self.pages, to_cuda(np.array(rows, np.int32)), st)
        codes = []
        for row in rows:
            ok = 0 <= row < len(self.table)
            codes.append(0 if ok else cb.ST_BAD_PAGES)
            if ok:
                for p in self.table[row][self.table[row] >= 0]:
                    self.ref[p] -= 1
                self.table[row] = -1
        self.check(st, codes, "free")

    def fork(self, src, dst, lengths):
        st = self.status(len(src))
        a = [to_cuda(np.array(x, np.int32)) for x in (src, dst, lengths)]
        cb.confu_pages_fork(self.ctx, self.dims, self.L, self.k, self.v, self.pages, *a, self.ws, st)
        codes, free, out, pairs, before = [], self.free_pages(), False, [], self.table.copy()
        for i, (s, d, n) in enumerate(zip(src, dst, lengths)):
            need, rows, width = -(-n // PAGE), len(self.table), self.table.shape[1]
            ok = 0 <= s < rows and 0 <= d < rows and 0 <= n <= width * PAGE and d not in dst[:i] and d not in src
            ok = ok and (before[s, :need] >= 0).all() and (before[d] < 0).all()
            if not ok:
                codes.append(cb.ST_BAD_PAGES)
            elif n % PAGE and (out or not free):
                out = True
                codes.append(cb.ST_NO_PAGES)
            else:
                codes.append(0)
                full = n // PAGE
                self.table[d, :full] = before[s, :full]
                for p in before[s, :full]:
                    self.ref[p] += 1
                if n % PAGE:
                    p = free.pop(0)
                    self.table[d, full], self.ref[p] = p, 1
                    pairs.append((int(before[s, full]), p))
        self.copy_pages(pairs)
        self.check(st, codes, "fork")

    def compact(self, with_map=True):
        used = H.guarded(self.regs, (1,), torch.int32, -1)
        page_map = H.guarded(self.regs, (self.n_pages,), torch.int32, -7) if with_map else None
        cb.confu_pages_compact(self.ctx, self.dims, self.L, self.k, self.v, self.pages, page_map, used, self.ws)
        n = int((self.ref > 0).sum())
        new = np.where(self.ref > 0, np.arange(self.n_pages), -1).astype(np.int32)
        holes = [p for p in range(n) if self.ref[p] == 0]
        pairs = [(p, holes.pop(0)) for p in range(n, self.n_pages) if self.ref[p] > 0]
        for p, q in pairs:
            new[p], self.ref[q], self.ref[p] = q, self.ref[p], 0
        self.table = np.where(self.table >= 0, new[np.maximum(self.table, 0)], -1).astype(np.int32)
        self.copy_pages(pairs)
        self.check(what="compact")
        assert used.tolist() == [n]
        if with_map:
            assert np.array_equal(page_map.cpu().numpy(), new)


@pytest.fixture()
def model(request):
    made = []

    def make(*a, **kw):
        made.append(Model(*a, **kw))
        return made[-1]
    yield make
    for m in made:
        m.close()


@pytest.mark.parametrize("kind,Hkv,D,block", [("bf16", 2, 64, 32), ("fp32", 1, 64, 32), ("fp8", 3, 128, 32), ("block", 2, 128, 32), ("block", 1, 64, 128)])
def test_a_life_of_a_pool(model, kind, Hkv, D, block):
    """Random requests in random order, refused ones among them."""
    m = model(37, 9, 6, seed=5 + D, kind=kind, Hkv=Hkv, D=D, block=block)
    r = m.r
    for turn in range(40):
        what = r.randint(0, 4)
        if what == 0:
            rows = list(r.randint(-1, 10, r.randint(1, 5)))
            m.reserve(rows, list(r.randint(-1, 6 * PAGE + 40, len(rows))))
        elif what == 1:
            m.free(list(r.randint(0, 10, r.randint(1, 3))))
        elif what == 2:
            empty = [i for i in range(9) if (m.table[i] < 0).all()]
            full = [i for i in range(9) if (m.table[i] >= 0).any()]
            if not full:
                continue
            n = r.randint(1, 4)
            src = list(r.choice(full, n))
            dst = list(r.choice(empty if empty and r.rand() < 0.8 else np.arange(9), n))
            m.fork(src, dst, [int(r.choice([(m.table[s] >= 0).sum() * PAGE, r.randint(0, (m.table[s] >= 0).sum() * PAGE + 1), r.randint(0, 6 * PAGE)])) for s in src])
        else:
            m.compact(with_map=bool(r.randint(0, 2)))
    m.free(list(range(9)))
    assert (m.ref == 0).all()


def test_refused_requests(model):
    m = model(6, 8, 4, seed=3)
    m.reserve([0, 0, 8, -1, 1, 2], [130, 130, 5, 5, 513, -1])        # a row twice, rows and lengths out of range
    m.reserve([1, 2, 3, 0], [256, 400, 1, 256])                      # four free pages: too few for row 2, nothing for row 3, row 0 has its own
    m.fork([0, 0, 1, 0, 5], [4, 4, 1, 0, 6], [256, 100, 100, 100, 10])       # named twice, a source, itself, a source without pages
    m.reserve([2], [200])
    m.fork([2, 2, 2], [5, 6, 7], [130, 128, 3])                      # no page left: the whole-page one is served all the same
    m.reserve([5, 6], [0, 0])
    m.free([2, 2, 5, 9])


@pytest.mark.parametrize("n_pages", [1, 3, 4097, 12289])
def test_pools_of_any_size(model, n_pages):
    m = model(n_pages, 3, max(2, n_pages // 2), seed=9, L=1, Hkv=1, D=64)
    m.reserve([0, 1], [n_pages // 2 * PAGE, 1])
    m.reserve([2], [(n_pages - n_pages // 2 - 1) // 2 * PAGE])
    m.free([0])
    m.compact()
    m.reserve([0], [PAGE])
    m.free([1])
    m.compact(with_map=False)
    m.compact()


def test_as_many_requests_as_a_call_takes(model):
    n = cb.MAX_PAGE_REQUESTS
    m = model(2 * n + 7, 2 * n, 3, seed=11, L=1, Hkv=1, D=128, kind="fp8")
    rows = list(m.r.permutation(n))
    m.reserve(rows, list(m.r.randint(0, 2 * PAGE, n)))
    full = [i for i in range(n) if m.table[i, 0] >= 0]
    dst = list(n + m.r.permutation(n))
    src = list(m.r.choice(full, n))
    m.fork(src, dst, [int(m.r.randint(0, (m.table[s] >= 0).sum() * PAGE + 1)) for s in src])
    m.free(rows)
    m.compact()
    with pytest.raises(cb.ConfuError) as e:
        cb.confu_pages_free(m.ctx, m.pages, torch.zeros(n + 1, dtype=torch.int32, device="cuda"))
    assert e.value.code == -5
    with pytest.raises(ValueError):
        cb.confu_pages_reserve(m.ctx, m.pages, torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"))


def test_copies_of_pages_and_ids_outside_the_pool(model):
    m = model(9, 1, 1, seed=13, kind="block")
    src, dst = [1, 8, 3, -1, 9, 2], [4, 5, 3, 6, 7, 9]
    st = m.status(6)
    cb.confu_pages_copy(m.ctx, m.dims, m.L, m.k, m.v, 9, to_cuda(np.array(src, np.int32)), to_cuda(np.array(dst, np.int32)), st)
    m.copy_pages([(1, 4), (8, 5)])
    m.check(st, [0, 0, 0, 12, 12, 12])


def test_calls_in_a_graph_and_on_a_stream(model):
    """A turn of a server, captured once and replayed: sequences end, others are continued twice, the pool is moved together."""
    m = model(40, 8, 4, seed=17, kind="block")
    m.reserve([0, 1, 2, 3], [500, 300, 200, 129])
    src, dst, lengths = (to_cuda(np.array(x, np.int32)) for x in ([0, 1, 1], [4, 5, 6], [400, 256, 140]))
    status, used = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

    def turn(stream):
        cb.confu_pages_free(m.ctx, m.pages, dst, status, stream)
        cb.confu_pages_fork(m.ctx, m.dims, m.L, m.k, m.v, m.pages, src, dst, lengths, m.ws, status, stream)
        cb.confu_pages_compact(m.ctx, m.dims, m.L, m.k, m.v, m.pages, None, used, m.ws, stream)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    turn(side)
    torch.cuda.synchronize()
    state = [m.d_table.clone(), m.d_ref.clone()] + [t.clone() for t in m.pools + m.scales]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn(torch.cuda.current_stream())
    graph.replay()
    torch.cuda.synchronize()
    for got, want in zip([m.d_table, m.d_ref] + m.pools + m.scales, state):      # the same sequences again: the same pages, where they were
        assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))
    assert status.tolist() == [0, 0, 0] and used.tolist() == [4 + 3 + 2 + 2 + 1 + 0 + 1]


def test_continuations_share_and_part_in_a_block_scaled_cache(model):
    """Two continuations of a sequence read its cache as it was, and write theirs apart."""
    from tests import block_ref as br
    Hkv, D, block = 2, 128, 32
    m = model(12, 4, 4, seed=19, kind="block", Hkv=Hkv, D=D, block=block, L=1)
    for t in m.scales:
        t.fill_(2.0 ** -7)
    for t in m.pools:
        t.copy_((torch.randn(t.shape, device="cuda") * 96).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    m.want = [t.clone() for t in m.pools + m.scales]
    m.reserve([0], [200])
    m.fork([0, 0], [1, 2], [200, 128])
    m.reserve([0, 1, 2], [203, 203, 131])
    cb.confu_set_paging(m.ctx, m.d_table, 4)
    cb.confu_set_kv_block_scales(m.ctx, m.scales[0], m.scales[1], None, None, block)
    P = np.array([200, 200, 128], np.int32)
    rows = torch.randn(3, 3, Hkv, D).bfloat16() * 64                 # scales grow
    dims = cb.make_dims(3, 4, Hkv, D, 3, 0, 0, cb.FP8_BLOCK)
    before = br.Cache(m.pools[0].cpu().numpy().copy(), m.scales[0].cpu().numpy().copy(), block, m.table)
    cb.confu_kv_append(m.ctx, dims, rows.cuda(), rows.cuda(), m.pools[0], m.pools[1], None, to_cuda(P))
    torch.cuda.synchronize()
    for b in range(3):
        before.append(b, int(P[b]), rows[b].double().numpy())
    assert np.array_equal(m.pools[0].cpu().numpy(), before.codes) and np.array_equal(m.scales[0].cpu().numpy(), before.scales)
    after = br.Cache(before.codes, before.scales, block, m.table)
    assert np.array_equal(after.read(0, range(192)), after.read(1, range(192)))       # up to the block that grew: the same entries
    assert np.array_equal(after.read(0, range(128)), after.read(2, range(128)))
    assert not np.array_equal(after.read(0, range(200, 203)), after.read(1, range(200, 203)))
