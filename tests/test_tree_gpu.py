"""Attention of a tree of drafted tokens against a plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

from tree_case import TreeCase, check

pytestmark = pytest.mark.gpu

GENERAL = 2  # FLAG_FORCE_GENERAL

FORMS = [("bf16", 128, 16), ("bf16", 128, 32), ("bf16", 64, 16), ("bf16", 64, 32), ("f8e4m3", 128, 32), ("f8e4m3", 128, 16),
         ("f8e4m3", 64, 32), ("f8e4m3", 64, 16), ("f32", 128, 16), ("f32", 64, 32), ("f32", 64, 16), ("f32", 128, 32)]


def verify_case(M, case, flags=0, want=None, **kw):
    got = case.run(M, flags, **kw)
    check(case, got, case.want() if want is None else want, M.last_kernel())
    return got


@pytest.mark.parametrize("flags", [0, GENERAL])
@pytest.mark.parametrize("masked,interleaved", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("kv_dtype,D,P", FORMS)
def test_every_form(mepic, kv_dtype, D, P, masked, interleaved, flags):
    case = TreeCase(11, [0, 1, 15, 16, 31, 33, 127, 130, 300, 517, 40], [5, 1, 3, 9, 16, 12, 7, 2, 11, 4, 0], D=D, P=P, kv_dtype=kv_dtype,
                    masked=masked, interleaved=interleaved, extra_tokens=3)
    verify_case(mepic, case, flags)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (12, 12), (32, 8), (28, 4), (5, 1), (16, 1), (48, 8), (32, 2)])
@pytest.mark.parametrize("kv_dtype", ["bf16", "f8e4m3", "f32"])
def test_heads_and_sizes_of_trees(mepic, kv_dtype, Hq, Hkv):
    """One node to 64, so that rows fill every tile and a little more."""
    for seed, nodes in ((1, [1, 1, 1]), (2, [2, 3, 1]), (3, [8, 5, 6]), (4, [17, 16, 15]), (5, [64, 33, 2])):
        case = TreeCase(seed, [200, 67, 391], nodes, Hq=Hq, Hkv=Hkv, P=32 if kv_dtype == "f8e4m3" else 16, kv_dtype=kv_dtype)
        verify_case(mepic, case)


@pytest.mark.parametrize("kv_dtype,D", [("bf16", 128), ("f8e4m3", 64), ("f32", 64)])
@pytest.mark.parametrize("chain", [False, True])
def test_largest_trees(mepic, kv_dtype, D, chain):
    """256 nodes, behind contexts that put node 0 anywhere in a group of slots; a chain of 256; many roots."""
    case = TreeCase(21, [45, 0, 97], [256, 255, 130], Hq=4, Hkv=2, D=D, kv_dtype=kv_dtype, parents="chain" if chain else "tree", spread=40,
                    roots=1 if chain else 9)
    verify_case(mepic, case)


@pytest.mark.parametrize("kv_dtype,Hq,Hkv", [("bf16", 8, 2), ("f8e4m3", 7, 1), ("f32", 2, 2)])
@pytest.mark.parametrize("ctx,nodes", [([9000], [6]), ([5000, 3, 2100, 700], [20, 1, 13, 5]), ([33000, 100], [3, 9])])
def test_contexts_cut_into_parts(mepic, kv_dtype, Hq, Hkv, ctx, nodes):
    case = TreeCase(31, ctx, nodes, Hq=Hq, Hkv=Hkv, P=32 if kv_dtype == "f8e4m3" else 16, kv_dtype=kv_dtype)
    verify_case(mepic, case)


def test_many_requests(mepic):
    """More requests than any workgroup has threads, some empty."""
    rng = np.random.default_rng(5)
    nodes = rng.integers(0, 5, 1400)
    case = TreeCase(41, rng.integers(0, 90, 1400), nodes, Hq=4, Hkv=2, D=64)
    verify_case(mepic, case)


def test_wide_tables_without_a_bound_on_the_lengths(mepic):
    """max_kv_len unknown: the table's width bounds the lengths, wherever they lie below it."""
    case = TreeCase(42, [700, 10, 95], [12, 3, 30])
    case.bt = np.pad(case.bt, ((0, 0), (0, 900)), constant_values=-1)
    a = verify_case(mepic, case)
    b = case.run(mepic, max_kv_len=int(case.kv.max()))
    assert np.allclose(a[: case.n], b[: case.n], rtol=0.02, atol=0.02)


@pytest.mark.parametrize("flags", [0, GENERAL])
@pytest.mark.parametrize("kv_dtype", ["bf16", "f8e4m3", "f32"])
def test_rows_that_see_nothing_are_zero(mepic, kv_dtype, flags):
    case = TreeCase(51, [70, 260, 33], [6, 9, 4], kv_dtype=kv_dtype, masked=True)
    case.bm[1] = 0
    for b, j in ((0, 2), (2, 0)):                             # a masked node is not seen by itself either
        n = int(case.ctx[b]) + j
        case.bm[b, n // case.P] &= np.uint32(~(1 << (n % case.P)) & 0xFFFFFFFF)
    got = verify_case(mepic, case, flags)
    assert (got[case.cu[1]: case.cu[2]] == 0).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("kv_dtype", ["bf16", "f8e4m3", "f32"])
def test_nodes_that_are_not_seen_may_hold_anything(mepic, kv_dtype, value):
    """Nodes off everybody's path (leaves) hold NaN or infinities: only their own rows may show it."""
    case = TreeCase(52, [70, 260, 33], [14, 9, 40], kv_dtype=kv_dtype)
    want = case.want()
    leaves = [(b, j) for b in range(3) for j in range(int(case.nodes[b])) if j not in case.parents[case.cu[b]: case.cu[b + 1]]]
    for b, j in leaves:
        page, slot = case.node_slot(b, j)
        case.fill(page, [slot], value if kv_dtype != "f8e4m3" else float("nan"))
    got = case.run(mepic)
    hit = np.array([case.cu[b] + j for b, j in leaves])
    assert np.isnan(got[hit]).all() or value == -float("inf")
    rest = np.setdiff1d(np.arange(case.n), hit)
    clean = got.copy()
    clean[hit] = want[0][hit]
    assert len(rest) and np.isfinite(got[rest]).all()
    check(case, clean, want, mepic.last_kernel())


def test_a_nan_in_the_context_is_in_every_row_of_its_head(mepic):
    case = TreeCase(53, [300, 80], [6, 5])
    page, slot = int(case.bt[0, 7]), 3
    case.pages.k[page, 1, :, slot, :] = float("nan")
    got = case.run(mepic).reshape(case.n, 2, 4, 128)
    assert np.isnan(got[:6, 1]).all() and np.isfinite(got[:6, 0]).all() and np.isfinite(got[6:]).all()


@pytest.mark.parametrize("kv_dtype,big", [("bf16", 5e3), ("bf16", 3e5), ("bf16", 1e30), ("f32", 1e30)])
def test_keys_beyond_half_precision(mepic, kv_dtype, big):
    """One dim of some keys is larger than fp16 holds; the queries are nought there but for one head, where the score decides alone."""
    case = TreeCase(54, [500, 90], [6, 9], kv_dtype=kv_dtype)
    X = 8 if kv_dtype == "bf16" else 4
    for page, slot, sign in ((int(case.bt[0, 3]), 5, 1), (int(case.bt[0, 20]), 11, -1), (int(case.bt[1, 2]), 0, -1)):
        case.pages.k[page, :, 127 // X, slot, 127 % X] = sign * big
    case.q[:, :, 127] = 0
    case.q[:, :, 63] = 0
    case.q[:, 3, 127] = 2.0 ** -10
    verify_case(mepic, case)


def test_scales_of_queries_and_keys_do_not_matter(mepic):
    """Queries times 2^20 and keys times 2^-20 and the other way round: the same scores."""
    for up in (20, -20, 60):
        case = TreeCase(55, [300, 41], [9, 5], kv_dtype="f32" if up == 60 else "bf16")
        case.pages.k *= 2.0 ** -(up if up != -20 else -4)
        case.q *= 2.0 ** (up if up != -20 else -4)
        if up == 20:
            case.pages.k *= 2.0 ** 10                        # (keys of 2^-10: small, above the smallest normal half)
            case.q *= 2.0 ** -10
        verify_case(mepic, case)


@pytest.mark.parametrize("spread", [4, 12])
@pytest.mark.parametrize("P", [16, 32])
def test_page_scales_over_many_decades(mepic, spread, P):
    case = TreeCase(56, [700, 90, 2000], [6, 9, 12], kv_dtype="f8e4m3", P=P, scale_spread=spread)
    want = case.want()
    verify_case(mepic, case, want=want)
    case.pages.v_scales[case.bt[1, 0]] = 0.0                  # a page of zeros
    verify_case(mepic, case)


def test_chains_are_trees_and_odd_parents_are_roots(mepic):
    case = TreeCase(61, [130, 77], [12, 30], parents="chain")
    a = case.run(mepic)
    case.parents = np.concatenate([np.arange(-1, T - 1) for T in case.nodes]).astype(np.int32)
    assert np.array_equal(case.run(mepic), a)
    case.parents[[3, 9, 20, 25]] = [3, 11, -9, 2 ** 31 - 1]   # itself, a later one, negative, out of range: roots
    verify_case(mepic, case)


def test_far_positions(mepic):
    for kv_dtype in ("bf16", "f32", "f8e4m3"):
        case = TreeCase(62, [200, 60], [6, 20], kv_dtype=kv_dtype, first_pos=0)
        case.bp = (np.arange(case.bt.shape[1])[None] * case.P + np.array([[500_000], [2_000_001]])).astype(np.int32)
        case.q_pos = (case.q_pos + np.repeat([500_000, 2_000_001], case.nodes)).astype(np.int32)
        case.bp[0, 5] = -40                                   # a chunk that lies elsewhere, before position 0
        verify_case(mepic, case)


@pytest.mark.parametrize("kv_dtype", ["bf16", "f32"])
def test_rows_at_any_element_of_a_buffer(mepic, kv_dtype):
    case = TreeCase(63, [130, 300], [5, 20], kv_dtype=kv_dtype)
    p = case.stage(mepic)
    mepic.attn_tree(p, case.dpar)
    want, n = case.out.clone(), case.dq.numel()
    for shift in (1, 3):
        q, out = (torch.full((n + 8,), 7.0, dtype=case.dq.dtype, device="cuda") for _ in range(2))
        q[shift: shift + n] = case.dq.flatten()
        p.q, p.out = (t.data_ptr() + shift * t.element_size() for t in (q, out))
        mepic.attn_tree(p, case.dpar)
        torch.cuda.synchronize()
        assert torch.equal(out[shift: shift + n], want.flatten()) and (out[:shift] == 7).all() and (out[shift + n:] == 7).all()


def test_more_nodes_than_promised_stay_in_bounds(mepic):
    """The rows of a request that breaks max_q_len mean nothing; the others are right, and nothing else is written."""
    case = TreeCase(64, [130, 300, 50], [5, 20, 6], extra_tokens=4)
    got, want = case.run(mepic, max_q_len=8), case.want()
    for b in (0, 2):
        rows = slice(case.cu[b], case.cu[b + 1])
        assert np.allclose(got[rows], want[0][rows], rtol=0.02, atol=0.02)
    assert (got[case.n:] == 7).all()


def test_fewer_slots_than_nodes(mepic):
    """Unspecified rows for that request, right ones for the next."""
    case = TreeCase(65, [0, 300], [40, 20])
    want = case.want()
    case.kv[0] = 3
    got = case.run(mepic)
    assert np.allclose(got[40:], want[0][40:], rtol=0.02, atol=0.02)


@pytest.mark.parametrize("given", [False, True])
def test_runs_on_its_stream(mepic, given):
    case = TreeCase(66, [130, 900], [5, 20])
    p = case.stage(mepic)
    mepic.attn_tree(p, case.dpar)
    want, q = case.out.clone(), case.dq.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    case.dq.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        case.dq.copy_(q)
        if not given:
            mepic.attn_tree(p, case.dpar)
    if given:
        mepic.attn_tree(p, case.dpar, stream=side)
    with torch.cuda.stream(side):
        got = case.out.clone()
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("kv_dtype", ["bf16", "f8e4m3", "f32"])
def test_captured_and_replayed_with_other_lengths(mepic, kv_dtype):
    """A graph of the call follows lengths, trees and tables on the device, and two graphs may share a workspace one after the other."""
    long = TreeCase(67, [900, 2000, 130], [16, 9, 12], kv_dtype=kv_dtype)
    p = long.stage(mepic)
    mepic.attn_tree(p, long.dpar)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mepic.attn_tree(p, long.dpar)
    want = long.want()
    for _ in range(3):
        long.out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        check(long, long.out.double().cpu().numpy(), want, mepic.last_kernel())
        eager = long.out.clone()
        mepic.attn_tree(p, long.dpar)
        torch.cuda.synchronize()
        assert torch.equal(long.out, eager)
    long.kv = (long.kv - 60).astype(np.int32)                 # shorter contexts; the nodes are the last slots again
    long.ctx -= 60
    long.dkv.copy_(torch.from_numpy(long.kv))
    long.out.fill_(7.0)
    g.replay()
    torch.cuda.synchronize()
    check(long, long.out.double().cpu().numpy(), long.want(), mepic.last_kernel())


def test_the_same_call_twice_gives_the_same_bits(mepic):
    case = TreeCase(68, [5000, 300, 2600], [16, 9, 60])
    a = case.run(mepic)
    for _ in range(3):
        assert np.array_equal(case.run(mepic), a)


def test_read_once_changes_nothing(mepic):
    for kv_dtype in ("bf16", "f8e4m3"):
        case = TreeCase(69, [900, 300], [16, 9], kv_dtype=kv_dtype)
        assert np.array_equal(case.run(mepic), case.run(mepic, mepic.FLAG_KV_READ_ONCE))
