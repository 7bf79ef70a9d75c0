"""The move of a kept path against the token-by-token definition: every byte of the pages equal."""
import ctypes

import numpy as np
import pytest
import torch

import workloads as W
from oracle import commit as oracle_commit
from oracle import verify

WORD = {"f32": np.uint32, "bf16": np.uint16, "f8e4m3": np.uint8}


def words(t):
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()]).numpy()


def code_values():
    return torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()


class Keep:
    def __init__(self, seed, firsts, nodes, *, kv_dtype="bf16", Hkv=2, D=128, P=16, share=None, kept=None):
        rng = self.rng = np.random.default_rng(seed)
        self.kv_dtype, self.P = kv_dtype, P
        B = len(firsts)
        self.first, self.nodes = np.array(firsts, np.int32), np.array(nodes, np.int32)
        nb = -(-(np.maximum(self.first, 0) + self.nodes) // P)
        total = int(nb.sum()) + 2
        ids = rng.permutation(total).astype(np.int32)
        self.bt = np.full((B, max(1, int(nb.max(initial=0)))), -1, np.int32)
        at = 0
        for b in range(B):
            self.bt[b, : nb[b]] = ids[at: at + nb[b]]
            at += int(nb[b])
        self.pages = W.gen_pages(seed, total, Hkv, P, D, kv_dtype)
        self.cu_tree = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
        paths = kept if kept is not None else [np.sort(rng.choice(T, rng.integers(0, T + 1), replace=False)) for T in nodes]
        self.kept = np.concatenate([np.asarray(p, np.int32) for p in paths] + [np.zeros(0, np.int32)]).astype(np.int32)
        self.cu_kept = np.concatenate([[0], np.cumsum([len(p) for p in paths])]).astype(np.int32)

    def want(self):
        k, v = words(self.pages.k).copy(), words(self.pages.v).copy()
        requant = None
        if self.kv_dtype == "f8e4m3":
            values = code_values()

            def requant(w, pf, pt, is_k):
                s = (self.pages.k_scales if is_k else self.pages.v_scales).numpy()
                if s[pf] == s[pt]:
                    return w
                with np.errstate(over="ignore", invalid="ignore"):
                    return oracle_commit.encode_e4m3((values[w] * s[pf]).astype(np.float32) / s[pt])
        lens = verify.kv_keep(k, v, self.bt, self.first, self.cu_tree, self.kept, self.cu_kept, P=self.P, requant=requant)
        return k, v, lens

    def stage(self, M):
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
        up = lambda t: None if t is None else t.cuda()  # noqa: E731
        self.k, self.v = self.pages.k.cuda(), self.pages.v.cuda()
        self.lens = torch.full((len(self.first),), -99, dtype=torch.int32, device="cuda")
        self.dev = [i32(a) for a in (self.bt, self.first, self.cu_tree, self.kept, self.cu_kept)]
        return M.make_keep_params(self.k, self.v, *self.dev, k_scales=up(self.pages.k_scales), v_scales=up(self.pages.v_scales), kv_lens_out=self.lens)

    def check(self):
        torch.cuda.synchronize()
        k, v, lens = self.want()
        assert np.array_equal(words(self.k.cpu()), k), "K"
        assert np.array_equal(words(self.v.cpu()), v), "V"
        assert self.lens.cpu().tolist() == [-99 if x is None else x for x in lens]


@pytest.mark.gpu
@pytest.mark.parametrize("D,P", [(128, 16), (128, 32), (64, 16), (64, 32)])
@pytest.mark.parametrize("kv_dtype", ["bf16", "f32", "f8e4m3"])
def test_kept_paths(mepic, kv_dtype, D, P):
    case = Keep(3, [0, 5, 31, 32, 100, -1, 77, 8], [1, 9, 26, 64, 256, 12, 200, 0], kv_dtype=kv_dtype, D=D, P=P)
    mepic.kv_keep(case.stage(mepic))
    case.check()


@pytest.mark.gpu
@pytest.mark.parametrize("Hkv", [1, 4, 12])
def test_overlapping_moves(mepic, Hkv):
    """Every slot is source and destination at once: the odd nodes, all but the first, all, none."""
    paths = [range(1, 200, 2), range(1, 200), range(200), [], range(150, 200), [199]]
    case = Keep(4, [3, 17, 40, 9, 64, 1], [200] * 6, Hkv=Hkv, kept=[list(p) for p in paths])
    mepic.kv_keep(case.stage(mepic))
    case.check()


@pytest.mark.gpu
@pytest.mark.parametrize("P", [16, 32])
def test_codes_take_the_scale_of_their_page(mepic, P):
    """Scales over many decades, equal ones, and values that saturate or vanish; NaN codes within a page."""
    case = Keep(5, [3, 16, 90, 14], [90, 64, 256, 40], kv_dtype="f8e4m3", P=P)
    for s in (case.pages.k_scales, case.pages.v_scales):
        s.copy_(torch.from_numpy(10.0 ** case.rng.uniform(-6, 6, s.numel()).round()).float())
    mepic.kv_keep(case.stage(mepic))
    case.check()


@pytest.mark.gpu
def test_entries_that_make_no_sense_are_left_out(mepic):
    paths = [[0, 4, 4, 9], [2, 1, 5, 8], [0, 3, 70, 6], [-3, 1, 2], [1, 2, 3], [0, 2 ** 31 - 1]]
    case = Keep(6, [3, 17, 40, 9, 30, 2], [10, 10, 10, 10, 10, 10], kept=paths)
    case.bt[4, 2] = 10 ** 6                                  # a page that does not exist
    mepic.kv_keep(case.stage(mepic))
    case.check()


@pytest.mark.gpu
def test_captured_and_replayed(mepic):
    """A graph follows paths on the device."""
    case = Keep(7, [3, 17, 100], [26, 12, 64])
    p = case.stage(mepic)
    mepic.kv_keep(p)
    case.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mepic.kv_keep(p)
    for seed in (1, 2, 3):
        rng = np.random.default_rng(seed)
        case.pages.k.copy_(case.k.cpu())
        case.pages.v.copy_(case.v.cpu())
        n = np.diff(case.cu_kept)
        case.kept = np.concatenate([np.sort(rng.choice(T, c, replace=False)) for T, c in zip(case.nodes, n)]).astype(np.int32)
        case.dev[3].copy_(torch.from_numpy(case.kept))
        g.replay()
        case.check()


@pytest.mark.gpu
def test_runs_on_its_stream(mepic):
    case = Keep(8, [3, 17, 100], [26, 12, 64])
    p = case.stage(mepic)
    k = case.k.clone()
    case.k.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        case.k.copy_(k)
    mepic.kv_keep(p, stream=side)
    side.synchronize()
    case.check()


# ------------------------------------------------------------------------------------------------ refusals (no GPU)
def test_refusals_before_any_launch(mepic):
    lib = mepic.load()
    here = 1 << 20

    def call(**over):
        p = mepic.KeepParams()
        base = dict(k_pages=here, v_pages=here, block_tables=here, first_slots=here, cu_tree=here, kept=here, cu_kept=here, B=2, n_kept=3, Hkv=2, D=128,
                    P=16, max_blocks=4, num_pages=9, kv_dtype=mepic.BF16)
        base.update(over)
        for k, v in base.items():
            setattr(p, k, v)
        return lib.mepic_kv_keep(ctypes.byref(p), None)
    for bad in (dict(k_pages=None), dict(v_pages=None), dict(block_tables=None), dict(first_slots=None), dict(cu_tree=None), dict(kept=None),
                dict(cu_kept=None), dict(B=-1), dict(n_kept=-1), dict(Hkv=0), dict(max_blocks=-1), dict(num_pages=-1), dict(kv_dtype=mepic.F8E4M3)):
        assert call(**bad) == mepic.ERR_INVALID, bad
    for bad in (dict(D=96), dict(P=8), dict(kv_dtype=7), dict(Hkv=70000)):
        assert call(**bad) == mepic.ERR_UNSUPPORTED, bad
    assert call(B=0) == mepic.OK
    assert lib.mepic_kv_keep(None, None) == mepic.ERR_INVALID


def test_the_binding_looks_at_types_and_shapes(mepic):
    i = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    k, v = torch.zeros(9, 2, 16, 16, 8, dtype=torch.bfloat16), torch.zeros(9, 2, 128, 16, dtype=torch.bfloat16)
    args = [k, v, i(3, 5), i(3), i(4), i(7), i(4)]
    for at, bad in ((0, k.float()), (0, k[:, :1]), (2, i(3, 5).long()), (3, i(4)), (4, i(3)), (6, i(3))):
        with pytest.raises(ValueError):
            mepic.make_keep_params(*args[:at], bad, *args[at + 1:])
    with pytest.raises(ValueError):
        mepic.make_keep_params(*args, kv_lens_out=i(2))
