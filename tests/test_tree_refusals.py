"""What attention of a tree refuses, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

HERE = 1 << 20  # never dereferenced on the host
POINTERS = ("q", "out", "k_pages", "v_pages", "block_tables", "kv_lens", "q_positions", "cu_q_lens", "workspace")


def params(M, **over):
    p = M.AttnParams()
    base = dict(B=2, n_q_tokens=20, Hq=8, Hkv=2, D=128, P=16, max_blocks=4, num_pages=8, max_q_len=12, q_dtype=M.BF16, kv_dtype=M.BF16,
                rope_theta=1e4, workspace_bytes=1 << 40, **dict.fromkeys(POINTERS, HERE))
    base.update(over)
    for k, v in base.items():
        setattr(p, k, v)
    return p


def test_refusals(mepic):
    call = lambda **o: mepic.load().mepic_attn_tree(ctypes.byref(params(mepic, **o)), None, None)  # noqa: E731
    for name in POINTERS[:-1]:
        assert call(**{name: None}) == mepic.ERR_INVALID, name
    for bad in (dict(B=0), dict(B=-1), dict(Hq=7), dict(n_q_tokens=-1), dict(rope_theta=0.0), dict(timing_start=HERE), dict(workspace=HERE + 8),
                dict(kv_dtype=mepic.F8E4M3)):
        assert call(**bad) == mepic.ERR_INVALID, bad
    for bad in (dict(D=96), dict(P=8), dict(Hq=68), dict(q_dtype=mepic.F32), dict(max_q_len=257, n_q_tokens=300), dict(max_q_len=0, n_q_tokens=300)):
        assert call(**bad) == mepic.ERR_UNSUPPORTED, bad
    assert call(n_q_tokens=0) == mepic.OK
    assert mepic.load().mepic_attn_tree(None, None, None) == mepic.ERR_INVALID
    assert mepic.load().mepic_attn_tree_workspace_size(ctypes.byref(params(mepic)), None) == mepic.ERR_INVALID


def test_workspace_size_and_the_binding(mepic):
    assert mepic.attn_tree_workspace_size(params(mepic)) >= 0
    with pytest.raises(mepic.MepicError) as e:
        mepic.attn_tree_workspace_size(params(mepic, max_q_len=300, n_q_tokens=400))
    assert e.value.status == mepic.ERR_UNSUPPORTED
    with pytest.raises(ValueError):
        mepic.attn_tree(params(mepic), torch.zeros(19, dtype=torch.int32))
    with pytest.raises(ValueError):
        mepic.attn_tree(params(mepic), torch.zeros(20, dtype=torch.int64))


def test_tables_wider_than_slots_can_be_numbered(mepic):
    call = lambda **o: mepic.load().mepic_attn_tree(ctypes.byref(params(mepic, **o)), None, None)  # noqa: E731
    assert call(max_blocks=1 << 27) == call(max_blocks=1 << 27, max_kv_len=100) == call(n_q_tokens=1 << 28, max_q_len=8) == mepic.ERR_UNSUPPORTED
    # the largest table that can be: the work of the matrix-core kernels still fits 32 bits for two requests, not for a thousand
    assert mepic.attn_tree_workspace_size(params(mepic, max_blocks=(1 << 27) - 1, max_kv_len=5000)) > 0
    assert mepic.attn_tree_workspace_size(params(mepic, max_blocks=(1 << 27) - 1, max_kv_len=5000, B=1000, n_q_tokens=8000)) == 0


def test_parents_elsewhere_or_of_another_kind(mepic):
    """The kernel would read whatever lies at a host address, or every other number: refused before the call."""
    for parents in (torch.zeros(20, dtype=torch.int32), torch.zeros(20), torch.zeros(4, 5, dtype=torch.int32), torch.zeros(40, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            mepic.attn_tree(params(mepic), parents)
