"""The verification calls as an engine uses them: pages and slots for a step's drafted tokens, commit, attention of the trees, the
accepted paths kept, and on with the lengths that come out, step after step, in one captured graph."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import verify
from tree_case import bound, random_tree, to_f64

pytestmark = pytest.mark.gpu


class Engine:
    """Five requests of some hundred slots on the GPU and, token by token, in numpy."""

    def __init__(self, M, kv_dtype, masked, seed=1):
        rng = self.rng = np.random.default_rng(seed)
        self.M, self.kv_dtype, self.masked = M, kv_dtype, masked
        self.Hq, self.Hkv, self.D, self.P = 8, 2, 128, 32 if kv_dtype == "f8e4m3" else 16
        self.B, self.most, self.theta = 5, 12, 5e5
        P, B = self.P, self.B
        self.len = rng.integers(1, 300, B)
        width = 40
        self.held = -(-self.len // P)
        self.num_pages = 220
        ids = rng.permutation(self.num_pages).astype(np.int32)
        self.bt = np.zeros((B, width), np.int32)
        at = 0
        for b in range(B):
            self.bt[b, : self.held[b]] = ids[at: at + self.held[b]]
            at += int(self.held[b])
        self.free, self.head = ids[at:], 0
        self.pages = W.gen_pages(seed, self.num_pages, self.Hkv, P, self.D, kv_dtype)
        self.bp = np.tile((np.arange(width) * P).astype(np.int32), (B, 1))
        self.bm = np.zeros((B, width), np.uint32)
        for b in range(B):
            for n in range(self.len[b]):
                self.bm[b, n // P] |= np.uint32(1 << (n % P))
        if masked:                                           # two pad slots in front, which are no positions either
            self.bm[:, 0] &= np.uint32(0xFFFFFFFC)
            self.bp -= 2
        self.pos = self.len - (2 if masked else 0)           # position of the next token
        self._stage()

    def _stage(self):
        M, B, n, dev = self.M, self.B, self.B * self.most, "cuda"
        src = torch.float32 if self.kv_dtype == "f32" else torch.bfloat16
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int32) if a.dtype.itemsize == 4 else a.astype(np.int32)).to(dev)  # noqa: E731
        up = lambda t: None if t is None else t.to(dev)  # noqa: E731
        e = lambda *k, dt=torch.int32: torch.zeros(k, dtype=dt, device=dev)  # noqa: E731
        d = self.d = dict(k=up(self.pages.k), v=up(self.pages.v), ks=up(self.pages.k_scales), vs=up(self.pages.v_scales), bt=i32(self.bt), kv=i32(self.len),
                          held=i32(self.held), free=i32(self.free), head=e(1), first=i32(self.pos), bp=i32(self.bp), bm=i32(self.bm), new=e(B),
                          depth=e(n), parents=e(n), kept=e(n), cu_kept=e(B + 1), kv_all=e(B), cu=e(B + 1), run=e(B), slot0=e(B), status=e(B),
                          q_pos=e(n), q=e(n, self.Hq, self.D, dt=src), out=e(n, self.Hq, self.D, dt=src),
                          k_new=e(n, self.Hkv, self.D, dt=src), v_new=e(n, self.Hkv, self.D, dt=src))
        masks = dict(block_positions=d["bp"], block_valid_mask=d["bm"]) if self.masked else {}
        make = lambda ws: M.make_extend_params(  # noqa: E731
            d["kv"], d["new"], d["bt"], P=self.P, num_pages=self.num_pages, kv_lens_out=d["kv_all"], cu_tokens=d["cu"], run_request=d["run"],
            run_first_slot=d["slot0"], status=d["status"], n_blocks=d["held"], n_blocks_out=d["held"], free_pages=d["free"], free_head=d["head"],
            free_head_out=d["head"], first_positions=d["first"], token_offsets=d["depth"], token_positions=d["q_pos"], workspace=ws, **masks)
        self.extend = make(e(max(256, M.tables_extend_workspace_size(make(None))), dt=torch.uint8))
        self.commit = M.make_commit_params(d["k_new"], d["v_new"], d["k"], d["v"], d["bt"], d["run"], d["slot0"], d["cu"], k_scales=d["ks"], v_scales=d["vs"])
        mk = lambda ws: M.make_params(  # noqa: E731
            d["q"], d["out"], d["k"], d["v"], d["bt"], d["kv_all"], d["q_pos"], rope_theta=self.theta, cu_q_lens=d["cu"], k_scales=d["ks"],
            v_scales=d["vs"], max_q_len=self.most, workspace=ws, **masks)
        self.attn = mk(e(max(256, M.attn_tree_workspace_size(mk(None))), dt=torch.uint8))
        self.keep = M.make_keep_params(d["k"], d["v"], d["bt"], d["slot0"], d["cu"], d["kept"], d["cu_kept"], k_scales=d["ks"], v_scales=d["vs"],
                                       kv_lens_out=d["kv"])

    def calls(self):
        self.M.tables_extend(self.extend)
        self.M.kv_commit(self.commit)
        self.M.attn_tree(self.attn, self.d["parents"])
        self.M.kv_keep(self.keep)

    def drafts(self):
        """This step's trees, values and accepted paths, put where the calls read them."""
        rng, B = self.rng, self.B
        T = rng.integers(0, self.most + 1, B)
        trees = [random_tree(rng, t) for t in T]
        paths = [verify.path_of(p, int(rng.integers(0, t)))[::-1] if t else [] for p, t in zip(trees, T)]
        self.T, self.trees, self.paths = T, trees, paths
        n = int(T.sum())
        put = lambda name, a: self.d[name][: len(a)].copy_(torch.from_numpy(np.asarray(a, np.int32)))  # noqa: E731
        put("new", T)
        put("parents", np.concatenate(trees))
        put("depth", np.concatenate([[len(verify.path_of(p, i)) - 1 for i in range(len(p))] for p in trees] + [[]]))
        put("kept", np.concatenate(paths + [[]]))
        put("cu_kept", np.concatenate([[0], np.cumsum([len(p) for p in paths])]))
        put("first", self.pos)
        self.vals = {k: torch.from_numpy(rng.standard_normal((n, h, self.D)).astype(np.float32)).to(self.d[k].dtype)
                     for k, h in (("q", self.Hq), ("k_new", self.Hkv), ("v_new", self.Hkv))}
        for k, v in self.vals.items():
            self.d[k].zero_()
            self.d[k][:n].copy_(v)
        self.d["out"].fill_(7.0)

    def check(self):
        """The step in numpy, held against what the calls left."""
        torch.cuda.synchronize()
        P, d, T = self.P, self.d, self.T
        w = verify.tables_extend(self.len, T, self.bt, P, num_pages=self.num_pages, n_blocks=self.held, free_pages=self.free, free_head=self.head,
                                 first_positions=self.pos, block_positions=self.bp, block_valid_mask=self.bm, max_tokens=self.B * self.most)
        assert w["status"] == [0] * self.B and d["status"].tolist() == w["status"]
        self.bt, self.held, self.head = w["block_tables"].astype(np.int32), np.array(w["n_blocks"]), w["free_head"]
        self.bp, self.bm = w["block_positions"].astype(np.int32), w["block_valid_mask"]
        assert np.array_equal(d["bt"].cpu().numpy(), self.bt) and d["held"].tolist() == list(self.held) and int(d["head"]) == self.head
        if self.masked:
            assert np.array_equal(d["bp"].cpu().numpy(), self.bp) and np.array_equal(d["bm"].cpu().numpy().view(np.uint32), self.bm)
        cu, n = np.array(w["cu"]), int(T.sum())
        # commit
        logical = [W.unpack_k(self.pages.k.float()), W.unpack_v(self.pages.v.float())]  # [page, H, P, D] as stored (codes for e4m3)
        stored = []
        for x, new, scales in zip(logical, ("k_new", "v_new"), (self.pages.k_scales, self.pages.v_scales)):
            vals = self.vals[new].float()
            for b in range(self.B):
                for i in range(T[b]):
                    s = int(self.len[b]) + i
                    page = int(self.bt[b, s // P])
                    y = vals[cu[b] + i]
                    if scales is not None:
                        y = (y / scales[page]).clamp(-448, 448).to(torch.float8_e4m3fn).float()
                    x[page, :, s % P] = y
            stored.append(x)
        dt = self.pages.k.dtype
        k_pages, v_pages = W.pack_k(stored[0], self.kv_dtype).to(dt), W.pack_v(stored[1]).to(dt)
        # attention
        depth = np.concatenate([[len(verify.path_of(p, i)) - 1 for i in range(len(p))] for p in self.trees] + [[]]).astype(np.int64)
        q_pos = np.repeat(self.pos, T) + depth
        n64 = lambda t: None if t is None else t.double().numpy()  # noqa: E731
        want = verify.tree_attention(self.vals["q"].double().numpy(), to_f64(k_pages, self.kv_dtype), to_f64(v_pages, self.kv_dtype), self.bt,
                                     self.len + T, q_pos, cu, np.concatenate(self.trees), theta=self.theta, k_scales=n64(self.pages.k_scales),
                                     v_scales=n64(self.pages.v_scales), block_positions=self.bp if self.masked else None,
                                     block_valid_mask=self.bm if self.masked else None)
        self.n, self.kv = n, self.len + T
        got = d["out"].double().cpu().numpy()
        assert (np.abs(got[:n] - want[0]) <= bound(self, want, self.M.last_kernel())).all()
        assert (got[n:] == 7).all()
        # the kept paths, token by token
        for x, scales in zip(stored, (self.pages.k_scales, self.pages.v_scales)):
            for b in range(self.B):
                for r, j in enumerate(self.paths[b]):
                    sf, st = int(self.len[b]) + j, int(self.len[b]) + r
                    pf, pt = int(self.bt[b, sf // P]), int(self.bt[b, st // P])
                    y = x[pf, :, sf % P].clone()
                    if scales is not None and scales[pf] != scales[pt]:
                        y = (y * scales[pf] / scales[pt]).clamp(-448, 448).to(torch.float8_e4m3fn).float()
                    x[pt, :, st % P] = y
        self.pages.k, self.pages.v = W.pack_k(stored[0], self.kv_dtype).to(dt), W.pack_v(stored[1]).to(dt)
        bits = lambda t: t.cpu().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])  # noqa: E731
        assert torch.equal(bits(d["k"]), bits(self.pages.k)) and torch.equal(bits(d["v"]), bits(self.pages.v))
        taken = np.array([len(p) for p in self.paths])
        self.len, self.pos = self.len + taken, self.pos + taken
        assert d["kv"].tolist() == self.len.tolist()


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("kv_dtype,masked", [("bf16", False), ("bf16", True), ("f8e4m3", False), ("f32", True)])
def test_steps_of_an_engine(mepic, kv_dtype, masked, captured):
    eng = Engine(mepic, kv_dtype, masked)
    eng.drafts()
    eng.calls()
    eng.check()
    run = eng.calls
    if captured:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            eng.calls()
        run = graph.replay
    for _ in range(6):
        eng.drafts()
        run()
        eng.check()
