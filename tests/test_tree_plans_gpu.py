"""Attention of a tree of drafted tokens where the plan of a call changes: row tiles by the largest and the mean request, rows on either side of every
tile, contexts that are cut and rows that are computed again behind a cut."""
import numpy as np
import pytest

from tree_case import TreeCase, check

pytestmark = pytest.mark.gpu


def verify_case(M, case, **kw):
    check(case, case.run(M, **kw), case.want(), M.last_kernel())


@pytest.mark.parametrize("kv_dtype", ["bf16", "f8e4m3", "f32"])
@pytest.mark.parametrize("nodes", [[8, 8, 8], [9, 1, 1], [16, 16], [17, 2, 1, 1], [32, 31], [33, 1, 1, 1], [33, 32, 30], [64, 60], [64, 9, 1, 1, 1, 1]])
def test_rows_of_a_tile(mepic, kv_dtype, nodes):
    """Four rows a node: 32, 64, 128 and 256 rows filled and exceeded, by all requests or by one of them."""
    P = 32 if kv_dtype == "f8e4m3" else 16
    ctx = [700 + 37 * i for i in range(len(nodes))]
    verify_case(mepic, TreeCase(71, ctx, nodes, Hq=8, Hkv=2, P=P, kv_dtype=kv_dtype))
    verify_case(mepic, TreeCase(72, ctx, nodes, Hq=8, Hkv=2, P=P, kv_dtype=kv_dtype, masked=True))


@pytest.mark.parametrize("kv_dtype", ["bf16", "f8e4m3", "f32"])
@pytest.mark.parametrize("ctx", [[505], [511, 3], [512], [520, 513], [1023], [4096, 17, 0, 2000]])
def test_contexts_around_the_first_cut(mepic, kv_dtype, ctx):
    case = TreeCase(73, ctx, [1] * len(ctx), Hq=4, Hkv=1, P=32 if kv_dtype == "f8e4m3" else 16, kv_dtype=kv_dtype)
    verify_case(mepic, case)
    verify_case(mepic, case, max_kv_len=int(case.kv.max()))


@pytest.mark.parametrize("masked,interleaved", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("D", [64, 128])
def test_cut_fp32(mepic, D, masked, interleaved):
    verify_case(mepic, TreeCase(74, [5000, 700, 0, 2111], [20, 5, 1, 3], Hq=12, Hkv=2, D=D, kv_dtype="f32", masked=masked, interleaved=interleaved,
                                extra_tokens=2))


@pytest.mark.parametrize("kv_dtype", ["bf16", "f8e4m3", "f32"])
def test_rows_computed_again_behind_a_cut(mepic, kv_dtype):
    """The last node of a tree holds NaN: it is in the partial of every row of its request, and only its own row may show it."""
    case = TreeCase(75, [6000, 90], [9, 4], P=32 if kv_dtype == "f8e4m3" else 16, kv_dtype=kv_dtype)
    want = case.want()
    page, slot = case.node_slot(0, 8)
    case.fill(page, [slot], float("nan"))
    got = case.run(mepic)
    assert np.isnan(got[8]).all()
    got[8] = want[0][8]
    check(case, got, want, mepic.last_kernel())
