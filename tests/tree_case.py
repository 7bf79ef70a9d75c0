"""Requests with a tree of drafted tokens behind their context, for the tests of the verification calls: lengths, trees and pages
from a seed, staged on the GPU for the library and kept in 64 bits for the oracle."""
import numpy as np
import torch

import workloads as W
from oracle import verify


def random_tree(rng, T, spread=4, roots=1):
    par = np.full(T, -1, np.int32)
    for i in range(roots, T):
        par[i] = rng.integers(max(0, i - spread), i)
    return par


def to_f64(t, kv_dtype):
    return t.double().numpy() if kv_dtype != "f8e4m3" else t.float().double().numpy()


class TreeCase:
    """ctx[b] context slots and nodes[b] nodes per request. Every request owns its pages, in shuffled order; pages nobody owns, slots
    behind a request's last one and, with `masked`, slots whose valid bit is 0 hold NaN."""

    def __init__(self, seed, ctx, nodes, *, Hq=8, Hkv=2, D=128, P=16, kv_dtype="bf16", theta=5e5, masked=False, interleaved=False,
                 parents="tree", spread=4, roots=1, extra_tokens=0, poison=True, scale_spread=0, first_pos=0):
        rng = self.rng = np.random.default_rng(seed)
        self.seed, self.Hq, self.Hkv, self.D, self.P, self.kv_dtype, self.theta = seed, Hq, Hkv, D, P, kv_dtype, theta
        self.interleaved = interleaved
        self.ctx, self.nodes = np.array(ctx, np.int64), np.array(nodes, np.int64)
        B = self.B = len(ctx)
        self.kv = (self.ctx + self.nodes).astype(np.int32)
        self.cu = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
        n = self.n = int(self.cu[-1])
        nb = -(-self.kv // P)
        width = max(1, int(nb.max()))
        total = int(nb.sum()) + 3
        ids = rng.permutation(total).astype(np.int32)
        self.bt = np.full((B, width), -7, np.int32)          # entries behind a request's last block are never looked at
        at = 0
        for b in range(B):
            self.bt[b, : nb[b]] = ids[at: at + nb[b]]
            at += int(nb[b])
        trees = [random_tree(rng, int(T), spread, roots) for T in nodes]
        self.parents = np.concatenate(trees + [np.zeros(0, np.int32)]).astype(np.int32) if parents == "tree" else None
        depth = []
        for b in range(B):
            par = trees[b] if self.parents is not None else np.arange(-1, int(nodes[b]) - 1)
            depth += [len(verify.path_of(par, i)) - 1 for i in range(int(nodes[b]))]
        self.bp = self.bm = None
        base = self.ctx.copy() + first_pos
        if masked:
            self.bm = rng.integers(1, 1 << P, (B, width), dtype=np.uint64).astype(np.uint32)
            self.bm[rng.random((B, width)) < 0.5] = (1 << P) - 1
            for b in range(B):                               # nodes are real tokens
                for s in range(int(self.ctx[b]), int(self.kv[b])):
                    self.bm[b, s // P] |= np.uint32(1 << (s % P))
            self.bp = (np.arange(width)[None] * P - rng.integers(0, 3, (B, width)).cumsum(1)).astype(np.int32)
            base = self.ctx - 2 * width
        self.q_pos = (np.repeat(base, self.nodes) + np.array(depth, dtype=np.int64)).astype(np.int32)
        used = np.zeros(total, bool)
        for b in range(B):
            used[self.bt[b, : nb[b]]] = True
        self.pages = W.gen_pages(seed, total, Hkv, P, D, kv_dtype, used=used if poison else None)
        if scale_spread:
            for s in (self.pages.k_scales, self.pages.v_scales):
                s.mul_(torch.from_numpy(10.0 ** rng.uniform(-scale_spread, 0, total)).float())
        if poison:
            for b in range(B):
                for j in range(int(nb[b])):
                    live = np.arange(j * P, (j + 1) * P) < self.kv[b]
                    if masked:
                        live &= ((int(self.bm[b, j]) >> np.arange(P)) & 1).astype(bool)
                    self.fill(int(self.bt[b, j]), np.flatnonzero(~live))
        self.extra = extra_tokens
        self.q = W.gen_q(seed, n + extra_tokens, Hq, D, "f32" if kv_dtype == "f32" else "bf16")

    def fill(self, page, slots, value=float("nan")):
        """Put a value into slots of a page (e4m3: its NaN code, or the code of the value)."""
        for t, k in ((self.pages.k, True), (self.pages.v, False)):
            for s in slots:
                at = (page, slice(None), slice(None), int(s))
                if self.kv_dtype == "f8e4m3":
                    code = 0x7F if value != value else int(torch.tensor(value).to(torch.float8_e4m3fn).view(torch.uint8))
                    t.view(torch.uint8)[at] = code
                else:
                    t[at] = value

    def node_slot(self, b, j):
        n = int(self.ctx[b]) + j
        return int(self.bt[b, n // self.P]), n % self.P

    def want(self):
        """(out, weighted mean of |v|, largest scale * sum |q k|), in 64 bits."""
        kd = self.kv_dtype
        n64 = lambda t: None if t is None else t.double().numpy()  # noqa: E731
        with np.errstate(invalid="ignore"):
            return verify.tree_attention(self.q[: self.n].double().numpy(), to_f64(self.pages.k, kd), to_f64(self.pages.v, kd), self.bt, self.kv,
                                         self.q_pos, self.cu, self.parents, theta=self.theta, k_scales=n64(self.pages.k_scales),
                                         v_scales=n64(self.pages.v_scales), block_positions=self.bp, block_valid_mask=self.bm,
                                         interleaved=self.interleaved)

    def stage(self, M, flags=0, max_kv_len=0, max_q_len=None):
        """The call's argument block; self.out is what it writes."""
        dev = torch.device("cuda:0")
        i32 = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a).view(np.int32)).to(dev)  # noqa: E731
        up = lambda t: None if t is None else t.to(dev)  # noqa: E731
        self.dq, self.out = up(self.q), torch.full(self.q.shape, 7.0, dtype=self.q.dtype, device=dev)
        self.dk, self.dv, self.dks, self.dvs = up(self.pages.k), up(self.pages.v), up(self.pages.k_scales), up(self.pages.v_scales)
        self.dbt, self.dkv, self.dcu, self.dpar, self.dpos = i32(self.bt), i32(self.kv), i32(self.cu), i32(self.parents), i32(
            np.concatenate([self.q_pos, np.zeros(self.extra, np.int32)]))
        if self.parents is not None and self.extra:
            self.dpar = torch.cat([self.dpar, self.dpar.new_zeros(self.extra)])
        flags |= M.FLAG_ROPE_INTERLEAVED if self.interleaved else 0
        make = lambda ws: M.make_params(  # noqa: E731
            self.dq, self.out, self.dk, self.dv, self.dbt, self.dkv, self.dpos, rope_theta=self.theta, cu_q_lens=self.dcu, k_scales=self.dks,
            v_scales=self.dvs, block_positions=i32(self.bp), block_valid_mask=i32(self.bm), flags=flags, max_kv_len=max_kv_len,
            max_q_len=int(self.nodes.max()) if max_q_len is None else max_q_len, workspace=ws)
        self.ws = torch.empty(max(256, M.attn_tree_workspace_size(make(None))), dtype=torch.uint8, device=dev).fill_(255)
        return make(self.ws)

    def run(self, M, flags=0, **kw):
        p = self.stage(M, flags, **kw)
        M.attn_tree(p, self.dpar)
        torch.cuda.synchronize()
        return self.out.double().cpu().numpy()


def bound(case, want, kernel):
    """How far a right result may be from `want`, element by element. `size` is scale * sum over pairs |q||k|, which bounds sum |q_i k_i| in any
    rotation. fp32 operands, sums of 128 products and phases of 1e-7 turns: 1e-5 of it in all. Matrix-core kernels on 16- and 8-bit
    pages: a key's element u c - w s has its cos and sin, its first product and its sum rounded to fp16, 2^-11 each of |u c| + |w s| <= |k| at
    most, so 3 sqrt(2) 2^-11 |k| for the pair; a query's pair 2^-11 |q|; together 5.25 x 2^-11 of `size`.
    A score that is off by d puts e^(2d) on weight over sum of weights; probabilities are rounded by 2^-8 (bf16) or less, sums of
    weights and of the products of 32 slots by 2^-24 a step; the result once to its own type."""
    out, mean, size = want
    f32 = case.kv_dtype == "f32"
    fine = f32 or kernel == "tree_general"
    d = size * (1e-5 if fine else 5.25 * 2.0 ** -11 + 1e-5)
    steps = (int(case.kv.max()) if fine else int(case.kv.max()) / 32 + 64) * 2.0 ** -24
    with np.errstate(over="ignore"):
        weight = np.expm1(2 * d)[..., None]
    rel = weight + (0 if fine else 2.0 ** -8) + steps + 2.0 ** -20
    return mean * rel + np.abs(out) * (2.0 ** -23 if f32 else 2.0 ** -8) + 1e-30


def check(case, got, want, kernel):
    """Every element within its bound, and the whole within what independent roundings add up to: the result's own
    and the probabilities' to bf16, at most 2^-8 / sqrt(3) of the norm each."""
    out = want[0]
    assert np.isfinite(got[: case.n]).all(), np.argwhere(~np.isfinite(got[: case.n]))[:4]
    over = np.abs(got[: case.n] - out) - bound(case, want, kernel)
    worst = np.unravel_index(over.argmax(), over.shape)
    assert over.max() <= 0, (kernel, worst, got[worst], out[worst], float(over.max()))
    if case.kv_dtype != "f32":
        off = np.linalg.norm(got[: case.n] - out) / max(np.linalg.norm(out), 1e-30)
        assert off <= 2 ** 0.5 * 2.0 ** -8 / 3 ** 0.5 * 1.15, off
    assert (got[case.n:] == 7).all()                         # rows behind the last request
