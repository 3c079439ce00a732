"""GPU parity of the block-scaled E4M3 cache (attention, append, compaction) with plain 64-bit forms (tests/block_ref.py).  Codes and
scales are equal to the bit; attention is within the tolerance derived there."""
import numpy as np
import pytest
import torch

from paper_2603_08899_b200 import binding as cb
from tests import block_ref as br
from tests import harness as H
from tests.block_ref import PAGE, to_cuda

pytestmark = pytest.mark.gpu


class Case:
    """A layer of a batch: what is not an entry of a sequence holds NaN codes and NaN scales."""

    def __init__(self, B=3, Hq=8, Hkv=2, D=128, T=20, C=6, S=4, block=64, prefix=(1, 400), seed=1, wide=0, odd_scales=False, rows_in=True):
        self.__dict__.update(B=B, Hq=Hq, Hkv=Hkv, D=D, T=T, C=C, S=S, R=T + C, block=block)
        r = self.r = np.random.RandomState(seed)
        self.P = np.array(prefix if isinstance(prefix, list) else r.randint(prefix[0], prefix[1] + 1, B), np.int32)
        self.n_pages, self.table = br.pages(self.P + self.R, r)
        self.parent, self.owner = br.tree(r, B, T, C)
        nb = PAGE // block

        def cache():
            codes = np.full((self.n_pages * PAGE, Hkv, D), 0x7f, np.uint8)
            scales = np.full((self.n_pages, Hkv, nb), np.nan, np.float32)
            c = br.Cache(codes, scales, block, self.table)
            for b in range(B):
                for p in range(0, int(self.P[b]) + (self.R if rows_in else 0)):
                    if p % block == 0:
                        c.scale(b, p)[:] = 2.0 ** r.randint(-8 - wide, -5 + wide, Hkv) * (r.uniform(0.6, 1.7, Hkv) if odd_scales else 1.0)
                    codes[c.slot(b, p)] = br.encode(r.randn(Hkv, D) * 96)
            return c
        self.k, self.v = cache(), cache()
        self.k_soft, self.v_soft = (br.encode(r.randn(S, Hkv, D) * 96) for _ in range(2))
        self.ks_soft, self.vs_soft = ((2.0 ** r.randint(-8, -5, (Hkv, nb))).astype(np.float32) for _ in range(2))
        self.q = (r.randn(B, self.R, Hq, D) * 2.0 ** r.randint(-3, 2, (B, self.R, Hq, 1))).astype(np.float32)
        self.q = torch.from_numpy(self.q).bfloat16().float().numpy()

    def want(self, sm_scale=None, weight_bits=8):
        sm = sm_scale or self.D ** -0.5
        outs = []
        for b in range(self.B):
            n = int(self.P[b]) + self.R
            at = np.arange(self.S) // self.block

            def with_soft(c, soft, scales):
                x = c.read(b, range(n))
                y = br.VALUES[soft] * scales[:, at].T[:, :, None].astype(np.float64)
                sc = np.concatenate([np.stack([c.scale(b, p) for p in range(n)]), scales[:, at].T]).astype(np.float64)
                return np.concatenate([x, y]), sc
            k, _ = with_soft(self.k, self.k_soft, self.ks_soft)
            v, vs = with_soft(self.v, self.v_soft, self.vs_soft)
            see = br.visible(int(self.P[b]), self.T, self.C, self.S, self.parent[b], self.owner[b])
            outs.append(br.attention(self.q[b].astype(np.float64), k, v, vs, see, sm, weight_bits))
        return [np.stack(x) for x in zip(*outs)]

    def device(self):
        d = dict(k=to_cuda(self.k.codes), v=to_cuda(self.v.codes), ks=to_cuda(self.k.scales), vs=to_cuda(self.v.scales), table=to_cuda(self.table),
                 P=to_cuda(self.P), parent=to_cuda(self.parent), owner=to_cuda(self.owner) if self.C else None, q=to_cuda(self.q).bfloat16())
        for n in ("k_soft", "v_soft", "ks_soft", "vs_soft"):
            d[n] = to_cuda(getattr(self, n)) if self.S else None
        return d

    def dims(self, sm_scale=0.0):
        return cb.make_dims(self.B, self.Hq, self.Hkv, self.D, self.T, self.C, self.S, cb.FP8_BLOCK, sm_scale)


@pytest.fixture()
def gpu():
    g = H.Gpu()
    yield g
    g.close()


def paths_of(gpu, case):
    """The kernels that take these sizes."""
    return [cb.ATTENTION_AUTO, cb.ATTENTION_TENSOR] + ([cb.ATTENTION_GENERIC] if case.R * case.Hq // case.Hkv <= (32 if case.D == 64 else 16) else [])


def attend(gpu, case, d, use_plan=True, sm_scale=0.0, stream=None):
    dims = case.dims(sm_scale)
    gpu.ensure_ws(dims)
    cb.confu_set_paging(gpu.ctx, d["table"], d["table"].shape[1])
    cb.confu_set_kv_block_scales(gpu.ctx, d["ks"], d["vs"], d["ks_soft"], d["vs_soft"], case.block)
    reg = []
    out = H.guarded(reg, d["q"].shape, torch.bfloat16, float("nan"))
    lse = H.guarded(reg, (case.B, case.R, case.Hq), torch.float32, float("nan"))
    status = H.guarded(reg, (case.B,), torch.int32, 0)
    plan = None
    if use_plan:
        plan = H.guarded(reg, (cb.confu_plan_bytes(gpu.ctx, dims),), torch.uint8)
        cb.confu_tree_plan(gpu.ctx, dims, None, d["P"], d["parent"], d["owner"], plan, status, stream)
    cb.confu_tree_attention(gpu.ctx, dims, d["q"], d["k"], d["v"], case.n_pages * PAGE, None, d["P"], d["k_soft"], d["v_soft"],
                            None if use_plan else d["parent"], None if use_plan else d["owner"], plan, out, lse, status, stream)
    torch.cuda.synchronize()
    H.assert_guards(reg, "attention over a block-scaled cache")
    assert gpu.ws_intact()
    return out.double().cpu().numpy(), lse.double().cpu().numpy(), status.cpu().numpy()


def compare(case, got, sm_scale=None, what=""):
    out, lse, tol, tol_lse = case.want(sm_scale)
    assert (got[2] == 0).all()
    assert np.isfinite(got[0]).all(), what
    worst = (np.abs(got[0] - out) / tol).max()
    assert worst <= 1, f"{what}: {worst} times the tolerance"
    worst = (np.abs(got[1] - lse) / tol_lse).max()
    assert worst <= 1, f"{what}: lse {worst} times the tolerance"


ATTEND = {
    "one_token": dict(T=1, C=0, S=0),
    "one_token_no_prefix": dict(T=1, C=0, S=0, prefix=[0, 1, 2]),
    "one_token_one_head": dict(T=1, C=0, S=0, Hq=1, Hkv=1, prefix=(100, 300)),
    "one_token_soft_owner": dict(T=1, C=1, S=1),
    "chain_g8": dict(T=5, C=1, S=16, Hq=16, Hkv=2, prefix=(1, 900), block=32),
    "rows_26": dict(),
    "rows_26_d64": dict(D=64, block=32),
    "rows_64_g4": dict(B=2, T=60, C=4, S=16, prefix=(130, 520), block=128),
    "rows_64_g4_d64": dict(B=2, T=60, C=4, S=16, prefix=(130, 520), D=64),
    "rows_128_two_groups": dict(B=2, T=64, C=64, S=16, block=32),
    "rows_100_d64_g4": dict(B=2, T=50, C=50, S=3, D=64),
    "g3": dict(Hq=6, Hkv=2, T=30, C=20),
    "g3_few": dict(Hq=6, Hkv=2, T=3, C=2),
    "g7_d64": dict(Hq=14, Hkv=2, T=9, C=2, D=64),
    "g32": dict(B=2, Hq=32, Hkv=1, T=12, C=4, block=32),
    "prefix_zero": dict(prefix=[0, 0, 0]),
    "ends_with_a_page": dict(T=12, C=4, prefix=[112, 240, 368]),
    "starts_a_page": dict(T=12, C=4, prefix=[128, 256, 127]),
    "soft_128": dict(S=128, block=32),
    "soft_33": dict(S=33, block=32),
    "long": dict(B=1, Hq=4, Hkv=1, T=4, C=1, prefix=[9000]),
    "long_tree": dict(B=1, Hq=4, Hkv=1, T=30, C=10, prefix=[6000]),
    "scales_apart": dict(wide=12, block=32, prefix=(200, 700)),
    "scales_apart_one_token": dict(T=1, C=0, S=0, wide=12, block=32, prefix=(200, 700)),
    "scales_not_powers_of_two": dict(odd_scales=True, block=32),
    "many_sequences": dict(B=40, Hq=4, Hkv=2, T=2, C=1, S=2, prefix=(0, 260)),
    "rows_28_d64": dict(D=64, T=5, C=2),
    "g32_d64": dict(B=2, D=64, Hq=32, Hkv=1, T=1, C=0, block=32),
    "rows_16": dict(T=3, C=1),
}


@pytest.mark.parametrize("name", ATTEND)
def test_attention(gpu, name):
    case = Case(seed=300 + list(ATTEND).index(name), **ATTEND[name])
    d = case.device()
    for path in paths_of(gpu, case):
        gpu.set_path(path)
        got = attend(gpu, case, d)
        compare(case, got, what=f"{name}, path {path}")
        again = attend(gpu, case, d, use_plan=False)                 # its own plan, and the same inputs: the same bits
        assert np.array_equal(got[0], again[0]) and np.array_equal(got[1], again[1])


# many stretches of several tiles for a CTA each: rings and barriers go round often
RUNS = {
    "one_token": dict(B=64, Hq=8, Hkv=8, T=1, C=0, S=0, prefix=(100, 900)),
    "one_token_g4_d64": dict(B=48, Hq=16, Hkv=4, D=64, T=1, C=0, S=4, prefix=(100, 900), block=32),
    "chain": dict(B=40, Hq=8, Hkv=4, T=9, C=2, S=4, prefix=(100, 900)),
    "trees": dict(B=40, Hq=8, Hkv=4, T=40, C=10, S=4, prefix=(100, 700)),
    "trees_two_tiles": dict(B=24, Hq=32, Hkv=8, T=40, C=10, S=4, prefix=(0, 500)),
    "trees_d64": dict(B=40, Hq=8, Hkv=4, D=64, T=40, C=10, S=4, prefix=(100, 700)),
    "thousands": dict(B=3001, Hq=2, Hkv=2, T=1, C=0, S=0, prefix=(0, 40)),
    "chain_d64": dict(B=40, Hq=8, Hkv=4, D=64, T=9, C=2, S=4, prefix=(100, 900)),
    "chain_16_rows": dict(B=40, Hq=8, Hkv=4, T=6, C=2, S=4, prefix=(100, 900)),
    "heads_30": dict(B=5, Hq=30, Hkv=30, T=2, C=1, S=2, prefix=(0, 500)),
    "heads_74": dict(B=5, Hq=74, Hkv=74, T=2, C=1, S=2, prefix=(0, 300)),
    "heads_200": dict(B=2, Hq=200, Hkv=200, T=2, C=1, S=2, prefix=(0, 300)),
}


@pytest.mark.parametrize("name", RUNS)
def test_attention_of_many_sequences(gpu, name):
    case = Case(seed=350 + list(RUNS).index(name), **RUNS[name])
    d = case.device()
    for path in paths_of(gpu, case):
        gpu.set_path(path)
        got = attend(gpu, case, d)
        compare(case, got, what=f"{name}, path {path}")
        for _ in range(5):
            again = attend(gpu, case, d)
            assert np.array_equal(got[0], again[0]) and np.array_equal(got[1], again[1])


@pytest.mark.parametrize("kw", [dict(T=3, C=1), dict(T=3, C=1, Hkv=1, Hq=4)])
def test_a_plan_for_the_other_kernel_is_refused(gpu, kw):
    """Nothing is written but the status."""
    case = Case(seed=45, **kw)
    d = case.device()
    dims = case.dims()
    gpu.ensure_ws(dims)
    cb.confu_set_paging(gpu.ctx, d["table"], d["table"].shape[1])
    cb.confu_set_kv_block_scales(gpu.ctx, d["ks"], d["vs"], d["ks_soft"], d["vs_soft"], case.block)
    for built, launched in ((cb.ATTENTION_GENERIC, cb.ATTENTION_TENSOR), (cb.ATTENTION_TENSOR, cb.ATTENTION_GENERIC)):
        gpu.set_path(built)
        reg = []
        plan = H.guarded(reg, (cb.confu_plan_bytes(gpu.ctx, dims),), torch.uint8)
        out = H.guarded(reg, d["q"].shape, torch.bfloat16, 7.0)
        lse = H.guarded(reg, (case.B, case.R, case.Hq), torch.float32, 7.0)
        status = H.guarded(reg, (case.B,), torch.int32, 0)
        cb.confu_tree_plan(gpu.ctx, dims, None, d["P"], d["parent"], d["owner"], plan, status)
        gpu.set_path(launched)
        cb.confu_tree_attention(gpu.ctx, dims, d["q"], d["k"], d["v"], case.n_pages * PAGE, None, d["P"], d["k_soft"], d["v_soft"], None, None, plan, out, lse,
                                status)
        torch.cuda.synchronize()
        H.assert_guards(reg, "refused plan")
        assert status.cpu().tolist() == [cb.ST_BAD_PLAN] * case.B
        assert (out == 7.0).all() and (lse == 7.0).all()


@pytest.mark.parametrize("T,C", [(1, 0), (3, 1), (30, 10)])
def test_a_plan_that_is_written_while_the_attention_is_on_its_way(gpu, T, C):
    """What is fetched ahead by the plan buffer's old contents is a hint, whatever they are."""
    case = Case(seed=46, T=T, C=C, S=0 if C == 0 else 4)
    d = case.device()
    dims = case.dims()
    want = attend(gpu, case, d)
    plan = torch.empty(cb.confu_plan_bytes(gpu.ctx, dims) // 4 + 1, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros_like(d["q"]), torch.zeros(case.B, case.R, case.Hq, device="cuda")
    status = torch.zeros(case.B, dtype=torch.int32, device="cuda")
    for fill in (-1, 0, 1, 0x7FFFFFFF, 0x7FFFFFFE, -2 ** 31):
        for _ in range(4):
            plan.fill_(fill)
            cb.confu_tree_plan(gpu.ctx, dims, None, d["P"], d["parent"], d["owner"], plan, status)
            cb.confu_tree_attention(gpu.ctx, dims, d["q"], d["k"], d["v"], case.n_pages * PAGE, None, d["P"], d["k_soft"], d["v_soft"], None, None, plan, out, lse,
                                    status)
        torch.cuda.synchronize()
        assert (status == 0).all()
        assert np.array_equal(out.double().cpu().numpy(), want[0]) and np.array_equal(lse.double().cpu().numpy(), want[1])


@pytest.mark.parametrize("T,C", [(3, 1), (30, 10)])
def test_entries_behind_four_gigabytes(gpu, T, C):
    """A pool of which the last pages alone are in use, past 2^32 bytes: append, attention, compaction and copies give what a small pool gives."""
    Hkv, D = 8, 128
    case = Case(Hq=8, Hkv=Hkv, T=T, C=C, prefix=[200, 60, 126], seed=47)
    page_bytes = PAGE * Hkv * D
    skip = 2 ** 32 // page_bytes + 3
    n_pages = skip + case.n_pages
    small, big = case.device(), case.device()
    for n in ("k", "v"):
        pool = torch.empty(n_pages * PAGE, Hkv, D, dtype=torch.uint8, device="cuda")
        pool[skip * PAGE:] = big[n]
        scales = torch.ones(n_pages, Hkv, PAGE // case.block, device="cuda")
        scales[skip:] = big[n + "s"]
        big[n], big[n + "s"] = pool, scales
    big["table"] = torch.where(big["table"] >= 0, big["table"] + skip, big["table"])
    rows = [torch.from_numpy(case.r.randn(case.B, case.R, Hkv, D).astype(np.float32)).bfloat16().cuda() for _ in range(2)]
    a, path = paths(case)
    dims = case.dims()
    gpu.ensure_ws(dims)
    results = []
    for d, first, total in ((small, 0, case.n_pages), (big, skip, n_pages)):
        ptrs = [torch.tensor([d[n].data_ptr()], dtype=torch.int64, device="cuda") for n in ("k", "v", "ks", "vs")]
        cb.confu_set_paging(gpu.ctx, d["table"], d["table"].shape[1])
        cb.confu_set_kv_block_scales(gpu.ctx, d["ks"], d["vs"], d["ks_soft"], d["vs_soft"], case.block)
        cb.confu_set_kv_block_scale_layers(gpu.ctx, ptrs[2], ptrs[3], case.block)
        cb.confu_kv_append(gpu.ctx, dims, rows[0], rows[1], d["k"], d["v"], None, d["P"])
        outs = []
        for kernel in paths_of(gpu, case):
            gpu.set_path(kernel)
            out = torch.zeros_like(d["q"])
            status = torch.zeros(case.B, dtype=torch.int32, device="cuda")
            cb.confu_tree_attention(gpu.ctx, dims, d["q"], d["k"], d["v"], total * PAGE, None, d["P"], d["k_soft"], d["v_soft"], d["parent"], d["owner"], None,
                                    out, None, status)
            torch.cuda.synchronize()
            assert (status == 0).all()
            outs.append(out)
        gpu.set_path(cb.ATTENTION_AUTO)
        new = torch.zeros(case.B, dtype=torch.int32, device="cuda")
        cb.confu_kv_compact(gpu.ctx, dims, 1, ptrs[0], ptrs[1], None, d["P"], to_cuda(a), to_cuda(path), new, status)
        used = sorted(set(case.table[case.table >= 0].tolist()))
        pair = [torch.tensor([first + used[i]], dtype=torch.int32, device="cuda") for i in (0, -1)]
        cb.confu_pages_copy(gpu.ctx, dims, 1, ptrs[0], ptrs[1], total, pair[0], pair[1], status[:1])
        torch.cuda.synchronize()
        assert (status == 0).all()
        results.append(outs + [d["k"][first * PAGE:], d["v"][first * PAGE:], d["ks"][first:], d["vs"][first:]])
    assert torch.isfinite(results[0][0].float()).all()
    for x, y in zip(*results):
        assert torch.equal(torch.nan_to_num(x.float()) if x.dtype == torch.float32 else x, torch.nan_to_num(y.float()) if y.dtype == torch.float32 else y)


def test_attention_with_another_scale_and_rows_of_any_size(gpu):
    case = Case(seed=41, T=6, C=2)
    case.q[0, 0] = 0.0                                               # equal weights
    case.q[1, 2] *= 2.0 ** -60
    case.q[2, 1] *= 2.0 ** 6                                         # one key takes it all
    d = case.device()
    for path in paths_of(gpu, case):
        gpu.set_path(path)
        compare(case, attend(gpu, case, d, sm_scale=0.03), sm_scale=0.03)


def test_pages_outside_the_pool_read_as_zeros_and_a_malformed_tree_as_a_status(gpu):
    case = Case(B=3, seed=43, prefix=[300, 300, 300], T=6, C=2, S=0)
    kept = case.table.copy()
    case.table[0, 1], case.table[1, 1] = case.n_pages, -1            # slots 128..255 of two sequences
    d = case.device()
    d["parent"][2, 3] = 5
    outs = {}
    for path in paths_of(gpu, case):
        gpu.set_path(path)
        out, lse, status = attend(gpu, case, d)
        assert list(status) == [0, 0, 1]
        assert (out[2] == 0).all() and (lse[2] == 0).all()
        outs[path] = out, lse
    case.table[:] = kept
    for b in range(2):
        page = int(kept[b, 1])
        case.k.codes[page * PAGE:(page + 1) * PAGE] = 0
        case.v.codes[page * PAGE:(page + 1) * PAGE] = 0
        case.k.scales[page] = case.v.scales[page] = 1
    want, want_lse, tol, tol_lse = case.want()
    for out, lse in outs.values():
        assert (np.abs(out[:2] - want[:2]) <= tol[:2]).all() and (np.abs(lse[:2] - want_lse[:2]) <= tol_lse[:2]).all()


@pytest.mark.parametrize("kw", [dict(T=6, C=2, S=20, prefix=[250, 60, 126]), dict(T=6, C=2, S=0, D=64, Hq=4, prefix=[250, 60, 126]),
                                dict(T=8, C=4, S=3, Hq=4, Hkv=2, prefix=[250, 60, 126]), dict(T=8, C=4, S=3, Hq=4, Hkv=2, D=64, prefix=[250, 60, 126]), dict(T=40, C=20, S=40, prefix=[250, 60, 126]),
                                dict(B=40, T=40, C=20, S=5, prefix=(0, 300), Hkv=4, Hq=16), dict(B=40, T=40, C=20, S=5, prefix=(0, 300), Hkv=4, Hq=16, D=64)])
def test_values_that_are_not_numbers_reach_the_rows_that_see_them_alone(gpu, kw):
    """NaN codes in keys and values of tree slots and soft prompts, a column of a value each: exactly the rows that see them, exactly that column."""
    case = Case(seed=51, **kw)
    r = case.r
    bad_v = np.zeros((case.B, case.T + case.C + case.S, case.Hkv, case.D), bool)
    bad_k = np.zeros((case.B, case.T + case.C + case.S, case.Hkv), bool)
    for b in range(case.B):
        for _ in range(3):
            j, h, d = r.randint(0, case.R), r.randint(0, case.Hkv), r.randint(0, case.D)
            case.v.codes[case.v.slot(b, int(case.P[b]) + j), h, d] = r.choice([0x7f, 0xff])
            bad_v[b, j, h, d] = True
        if b % 2:
            j, h = r.randint(case.R // 2, case.R), r.randint(0, case.Hkv)
            case.k.codes[case.k.slot(b, int(case.P[b]) + j), h, 5] = 0x7f
            bad_k[b, j, h] = True
    if case.S:
        case.v_soft[case.S - 1, 0, 7] = 0xff
        bad_v[:, case.R + case.S - 1, 0, 7] = True
    want = np.zeros((case.B, case.R, case.Hq, case.D), bool)
    G = case.Hq // case.Hkv
    for b in range(case.B):
        see = br.visible(int(case.P[b]), case.T, case.C, case.S, case.parent[b], case.owner[b])[:, int(case.P[b]):]
        for h in range(case.Hq):
            want[b, :, h] = (see @ bad_v[b, :, h // G].astype(int) > 0) | (see @ bad_k[b, :, h // G].astype(int) > 0)[:, None]
    d = case.device()
    # numbers in their places: what the rows that do not see them, and their other columns, are
    case.v.codes[(case.v.codes & 127) == 127] = 0
    case.k.codes[(case.k.codes & 127) == 127] = 0
    case.v_soft[(case.v_soft & 127) == 127] = 0
    out, _, tol, _ = case.want()
    for path in paths_of(gpu, case):
        gpu.set_path(path)
        got, lse, status = attend(gpu, case, d)
        assert (status == 0).all()
        assert np.array_equal(np.isnan(got), want), f"path {path}"
        fine = ~want
        assert (np.abs(got[fine] - out[fine]) <= tol[fine]).all(), f"path {path}"


# ------------------------------------------------------------------------------------------------ writing
def layers(case, n, seed):
    r = np.random.RandomState(seed)
    return [(br.Cache(r.permutation(case.k.codes), case.k.scales * 2.0 ** r.randint(-1, 2), case.block, case.table),
             br.Cache(case.v.codes.copy(), case.v.scales.copy(), case.block, case.table)) for _ in range(n)]


def same(got, want, what):
    got = got.cpu().numpy()
    assert got.dtype == want.dtype and np.array_equal(got, want, equal_nan=got.dtype.kind == "f"), what


APPEND = {
    "one_row": dict(T=1, C=0),
    "one_row_no_prefix": dict(T=1, C=0, prefix=[0, 128, 127]),
    "rows_26_block_32": dict(block=32),
    "rows_26_block_128": dict(block=128),
    "rows_128": dict(T=64, C=64, block=32, prefix=(0, 300)),
    "rows_128_block_128_d64": dict(T=64, C=64, block=128, D=64, prefix=(0, 300)),
    "starts_a_block": dict(block=64, prefix=[64, 128, 192]),
    "last_slot_of_a_block": dict(block=64, prefix=[63, 127, 191]),
    "head_dim_64": dict(D=64, block=32, Hkv=3, Hq=3),
}


@pytest.mark.parametrize("size", [-6, 0, 5])
@pytest.mark.parametrize("name", APPEND)
def test_append(gpu, name, size):
    """size: the rows' magnitude against the cached entries', as a power of two: scales stay or grow."""
    case = Case(seed=500 + list(APPEND).index(name), rows_in=False, **APPEND[name])
    r = case.r
    d = case.device()
    rows = [torch.from_numpy((r.randn(case.B, case.R, case.Hkv, case.D) * 2.0 ** (size + r.randint(-3, 1, (case.B, case.R, case.Hkv, 1)))).astype(np.float32)).bfloat16()
            for _ in range(2)]
    cb.confu_set_paging(gpu.ctx, d["table"], d["table"].shape[1])
    cb.confu_set_kv_block_scales(gpu.ctx, d["ks"], d["vs"], None, None, case.block)
    for _ in range(2):                                               # a second time: the same again
        cb.confu_kv_append(gpu.ctx, case.dims(), rows[0].cuda(), rows[1].cuda(), d["k"], d["v"], None, d["P"])
    torch.cuda.synchronize()
    for c, x in ((case.k, rows[0]), (case.v, rows[1])):
        for b in range(case.B):
            c.append(b, int(case.P[b]), x[b].double().numpy())
    for n, want in (("k", case.k.codes), ("v", case.v.codes), ("ks", case.k.scales), ("vs", case.v.scales)):
        same(d[n], want, n)


@pytest.mark.parametrize("was", [1.0, 0.75])
def test_every_code_is_encoded_again_for_every_larger_scale(gpu, was):
    """All codes as prefix entries of a block whose scale grows 2^0 .. 2^39 times: each is the nearest code of its value."""
    n = 40
    case = Case(B=n, Hq=1, Hkv=1, T=1, C=0, S=0, prefix=[2] * n, block=32, rows_in=False, seed=63)
    rows = torch.zeros(n, 1, 1, 128, dtype=torch.bfloat16)
    for b in range(n):
        for c in (case.k, case.v):
            c.scale(b, 0)[:] = was
            c.codes[c.slot(b, 0), 0], c.codes[c.slot(b, 1), 0] = np.arange(128), np.arange(128, 256)
        rows[b] = 448.0 * 2.0 ** b
    d = case.device()
    cb.confu_set_paging(gpu.ctx, d["table"], d["table"].shape[1])
    cb.confu_set_kv_block_scales(gpu.ctx, d["ks"], d["vs"], None, None, case.block)
    cb.confu_kv_append(gpu.ctx, case.dims(), rows.cuda(), rows.cuda(), d["k"], d["v"], None, d["P"])
    torch.cuda.synchronize()
    for b in range(n):
        case.k.append(b, 2, rows[b].double().numpy())
        assert case.k.scale(b, 0)[0] == max(was, 2.0 ** b)
    same(d["ks"], case.k.scales, "scales")
    got, want = d["k"].cpu().numpy(), case.k.codes
    nan = (want & 127) == 127
    assert np.array_equal((got & 127) == 127, nan) and np.array_equal(got[~nan], want[~nan])


def test_append_of_rows_that_are_not_numbers(gpu):
    case = Case(B=2, T=5, C=0, prefix=[40, 0], block=32, rows_in=False, seed=61)
    rows = torch.from_numpy(case.r.randn(2, 5, 2, 128).astype(np.float32)).bfloat16()
    rows[0, 1, 0, 3] = float("inf")
    rows[0, 2, 1, 5] = -float("inf")
    rows[1, 0] = float("nan")
    rows[1, 1] = 0.0
    rows[1, 2, :, :64] = 3e38
    rows[1, 3] = 1e-38
    d = case.device()
    cb.confu_set_paging(gpu.ctx, d["table"], d["table"].shape[1])
    cb.confu_set_kv_block_scales(gpu.ctx, d["ks"], d["vs"], None, None, case.block)
    for x, n in ((rows, 5), (torch.zeros_like(rows), 5)):
        cb.confu_kv_append(gpu.ctx, case.dims(), x.cuda(), x.cuda(), d["k"], d["v"], None, d["P"])
        torch.cuda.synchronize()
        for b in range(2):
            case.k.append(b, int(case.P[b]), x[b].double().numpy())
        same(d["ks"], case.k.scales, "scales")
        got = d["k"].cpu().numpy()
        nan = (got & 127) == 127
        assert np.array_equal(nan, (case.k.codes & 127) == 127)
        assert np.array_equal(got[~nan], case.k.codes[~nan])


def paths(case, most=None):
    a = np.zeros(case.B, np.int32)
    path = np.full((case.B, 64), -1, np.int32)
    for b in range(case.B):
        a[b] = case.r.randint(0, (most or case.T - 1) + 1) if case.T > 1 else 0
        path[b, 0] = 0
        path[b, 1:a[b] + 1] = np.sort(case.r.permutation(np.arange(1, case.T))[:a[b]])
    return a, path


@pytest.mark.parametrize("block,D,T,wide", [(32, 128, 64, 0), (32, 64, 64, 6), (64, 128, 40, 6), (128, 64, 20, 4), (128, 128, 64, 6), (32, 128, 1, 0)])
def test_compaction_of_all_layers(gpu, block, D, T, wide):
    case = Case(B=5, T=T, C=3, D=D, block=block, wide=wide, prefix=[0, 1, 127, 200, 31], seed=71 + block)
    n = 3
    ls = []
    for i in range(n):
        c = Case(B=5, T=T, C=3, D=D, block=block, wide=wide, prefix=[0, 1, 127, 200, 31], seed=71 + block)
        for x in (c.k, c.v):
            x.table = case.table
            x.scales *= 2.0 ** i
        ls.append(c)
    a, path = paths(case)
    a[1], path[1, :3], path[1, 3:] = 0, [0, -1, -1], -1
    dev = [(to_cuda(c.k.codes), to_cuda(c.v.codes), to_cuda(c.k.scales), to_cuda(c.v.scales)) for c in ls]
    ptrs = [torch.tensor([x[i].data_ptr() for x in dev], dtype=torch.int64, device="cuda") for i in range(4)]
    table, P = to_cuda(case.table), to_cuda(case.P)
    cb.confu_set_paging(gpu.ctx, table, table.shape[1])
    cb.confu_set_kv_block_scale_layers(gpu.ctx, ptrs[2], ptrs[3], block)
    new, status = torch.full((5,), -7, dtype=torch.int32, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
    cb.confu_kv_compact(gpu.ctx, case.dims(), n, ptrs[0], ptrs[1], None, P, to_cuda(a), to_cuda(path), new, status)
    torch.cuda.synchronize()
    assert (status == 0).all()
    assert np.array_equal(new.cpu().numpy(), case.P + a + 1)
    for c, x in zip(ls, dev):
        for b in range(5):
            c.k.compact(b, int(case.P[b]), int(a[b]), path[b])
            c.v.compact(b, int(case.P[b]), int(a[b]), path[b])
        for got, want, what in zip(x, (c.k.codes, c.v.codes, c.k.scales, c.v.scales), ("k", "v", "ks", "vs")):
            same(got, want, what)


def test_compaction_refuses_paths_that_are_not_chains(gpu):
    case = Case(B=4, T=8, C=0, prefix=[5, 60, 128, 0], seed=81)
    path = np.full((4, 64), -1, np.int32)
    path[0, :3] = [0, 3, 3]
    path[1, :3] = [0, 2, 8]
    path[2, :2] = [1, 2]
    path[3, :3] = [0, 1, 5]
    a = np.array([2, 2, 1, 2], np.int32)
    d = case.device()
    k, v, ks, vs = (torch.tensor([d[n].data_ptr()], dtype=torch.int64, device="cuda") for n in ("k", "v", "ks", "vs"))
    cb.confu_set_paging(gpu.ctx, d["table"], d["table"].shape[1])
    cb.confu_set_kv_block_scale_layers(gpu.ctx, ks, vs, case.block)
    new, status = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    cb.confu_kv_compact(gpu.ctx, case.dims(), 1, k, v, None, d["P"], to_cuda(a), to_cuda(path), new, status)
    torch.cuda.synchronize()
    assert status.tolist() == [cb.ST_BAD_PATH] * 3 + [0]
    assert new.tolist() == [6, 61, 129, 3]
    case.k.compact(3, 0, 2, path[3])
    same(d["k"], case.k.codes, "k")
    same(d["ks"], case.k.scales, "ks")


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("T,C,block,D", [(1, 0, 32, 128), (9, 3, 64, 128), (40, 10, 32, 64)])
def test_steps_of_append_attention_and_compaction(gpu, T, C, block, D):
    """Three steps from empty prefixes of which two grow past a page: appended, attended, the accepted path kept; once eagerly on a stream of
    its own, once captured into a graph and replayed."""
    B = 3
    case = Case(B=B, T=T, C=C, S=0, D=D, block=block, prefix=[0, 126, 200], seed=91 + T, rows_in=False)
    case.n_pages, case.table = br.pages(np.array([300, 400, 500]), case.r)
    nb = PAGE // block
    for name in ("k", "v"):
        old = getattr(case, name)
        new = br.Cache(np.full((case.n_pages * PAGE, case.Hkv, D), 0x7f, np.uint8), np.full((case.n_pages, case.Hkv, nb), np.nan, np.float32), block, case.table)
        for b in range(B):
            if case.P[b]:
                new.append(b, 0, case.r.randn(int(case.P[b]), case.Hkv, D))
        setattr(case, name, new)
        del old
    d = case.device()
    dims = case.dims()
    gpu.ensure_ws(dims)
    side, graph = torch.cuda.Stream(), None
    rows = [torch.empty(B, case.R, case.Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    out = torch.empty_like(d["q"])
    plan = torch.empty(cb.confu_plan_bytes(gpu.ctx, dims), dtype=torch.uint8, device="cuda")
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    new_P = torch.empty_like(d["P"])
    acc, path_d = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, 64, dtype=torch.int32, device="cuda")
    ptrs = [torch.tensor([d[n].data_ptr()], dtype=torch.int64, device="cuda") for n in ("k", "v", "ks", "vs")]
    cb.confu_set_paging(gpu.ctx, d["table"], d["table"].shape[1])
    cb.confu_set_kv_block_scales(gpu.ctx, d["ks"], d["vs"], None, None, block)
    cb.confu_set_kv_block_scale_layers(gpu.ctx, ptrs[2], ptrs[3], block)

    def step(stream):
        cb.confu_tree_plan(gpu.ctx, dims, None, d["P"], d["parent"], d["owner"], plan, status, stream)
        cb.confu_kv_append(gpu.ctx, dims, rows[0], rows[1], d["k"], d["v"], None, d["P"], stream)
        cb.confu_tree_attention(gpu.ctx, dims, d["q"], d["k"], d["v"], case.n_pages * PAGE, None, d["P"], None, None, None, None, plan, out, None, status, stream)
        cb.confu_kv_compact(gpu.ctx, dims, 1, ptrs[0], ptrs[1], None, d["P"], acc, path_d, new_P, status, stream)
        with torch.cuda.stream(stream):
            d["P"].copy_(new_P)
    for i in range(3):
        x = [torch.from_numpy((case.r.randn(B, case.R, case.Hkv, D) * 2.0 ** (2 * i - 2)).astype(np.float32)).bfloat16() for _ in range(2)]
        a, path = paths(case, min(5, T - 1) if T > 1 else None)
        for to, src in zip(rows, x):
            to.copy_(src)
        acc.copy_(torch.from_numpy(a))
        path_d.copy_(torch.from_numpy(path))
        torch.cuda.synchronize()
        if i < 2:
            step(side)
        else:
            before = {n: d[n].clone() for n in ("k", "v", "ks", "vs", "P")}
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step(torch.cuda.current_stream())
            for n, t in before.items():
                d[n].copy_(t)
            graph.replay()
        torch.cuda.synchronize()
        for b in range(B):
            case.k.append(b, int(case.P[b]), x[0][b].double().numpy())
            case.v.append(b, int(case.P[b]), x[1][b].double().numpy())
        want, _, tol, _ = case.want()
        assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
        for b in range(B):
            case.k.compact(b, int(case.P[b]), int(a[b]), path[b])
            case.v.compact(b, int(case.P[b]), int(a[b]), path[b])
        case.P = case.P + a + 1
        assert np.array_equal(d["P"].cpu().numpy(), case.P)
        for n, c in (("k", case.k), ("v", case.v)):
            same(d[n], c.codes, n)
            same(d[n + "s"], c.scales, n + "s")
        assert (status == 0).all()
