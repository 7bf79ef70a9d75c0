"""Tables, slot maps and positions of a step's new tokens against the request-by-request definition: every entry equal."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import verify


class Step:
    def __init__(self, seed, B, P, *, new_hi, held_hi=20, pages=True, masks=False, offsets=False, short=0, spare=5, room=3, width=None, first=True,
                 head=0):
        rng = self.rng = np.random.default_rng(seed)
        self.B, self.P = B, P
        self.kv = rng.integers(0, held_hi * P + 1, B).astype(np.int32)
        self.new = rng.integers(0, new_hi + 1, B).astype(np.int32)
        self.held = (-(-self.kv // P) + (rng.random(B) < 0.4)).astype(np.int32)
        need = np.maximum(0, -(-(self.kv + self.new) // P) - self.held)
        self.width = int((-(-(self.kv + self.new) // P)).max(initial=0)) + 2 if width is None else width
        self.num_pages = int(self.held.sum() + need.sum()) + spare + head + 1
        ids = rng.permutation(self.num_pages).astype(np.int32)
        self.bt = rng.choice(ids, (B, self.width)).astype(np.int32) if B else np.zeros((0, self.width), np.int32)
        self.free = ids[: max(0, head + int(need.sum()) + spare - short)] if pages else None
        self.head, self.pages, self.masks = head, pages, masks
        self.first = rng.integers(-50, 1000, B).astype(np.int32) if first else None
        self.room = int(np.maximum(self.new, 0).sum()) + room
        self.offsets = rng.integers(0, 9, self.room).astype(np.int32) if offsets else None
        self.bp = rng.integers(-9, 999, (B, self.width)).astype(np.int32) if masks else None
        self.bm = rng.integers(0, 1 << 32, (B, self.width), dtype=np.uint64).astype(np.uint32) if masks else None

    def want(self):
        return verify.tables_extend(self.kv, self.new, self.bt, self.P, num_pages=self.num_pages, n_blocks=self.held if self.pages else None,
                                    free_pages=self.free, free_head=self.head, first_positions=self.first, token_offsets=self.offsets,
                                    block_positions=self.bp, block_valid_mask=self.bm, max_tokens=self.room)

    def run(self, M, in_place=False, tokens=True):
        dev = torch.device("cuda:0")
        up = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a).view(np.int32)).to(dev)  # noqa: E731
        e = lambda n, dt=torch.int32: torch.full((n,), -99, dtype=dt, device=dev)  # noqa: E731
        B = self.B
        d = self.d = dict(kv=up(self.kv), new=up(self.new), bt=up(self.bt), first=up(self.first), offsets=up(self.offsets), bp=up(self.bp), bm=up(self.bm))
        kw = {}
        if self.pages:
            d.update(held=up(self.held), free=up(self.free), head=torch.tensor([self.head], dtype=torch.int32, device=dev))
            d["held_out"], d["head_out"] = (d["held"], d["head"]) if in_place else (e(B), e(1))
            kw = dict(n_blocks=d["held"], n_blocks_out=d["held_out"], free_pages=d["free"], free_head=d["head"], free_head_out=d["head_out"])
        d["kv_out"] = d["kv"] if in_place else e(B)
        d.update(cu=e(B + 1), run=e(B), slot0=e(B), status=e(B))
        if tokens:
            d.update(slots=e(self.room, torch.int64), positions=e(self.room), requests=e(self.room))
        make = lambda ws: M.make_extend_params(  # noqa: E731
            d["kv"], d["new"], d["bt"], P=self.P, num_pages=self.num_pages, kv_lens_out=d["kv_out"], cu_tokens=d["cu"], run_request=d["run"],
            run_first_slot=d["slot0"], status=d["status"], first_positions=d["first"], token_offsets=d["offsets"], token_slots=d.get("slots"),
            token_positions=d.get("positions"), token_requests=d.get("requests"), block_positions=d["bp"], block_valid_mask=d["bm"],
            max_tokens=self.room, workspace=ws, **kw)
        ws = torch.full((max(256, M.tables_extend_workspace_size(make(None))),), 255, dtype=torch.uint8, device=dev)
        self.params = make(ws)
        M.tables_extend(self.params)
        torch.cuda.synchronize()
        return {k: v.cpu().numpy() for k, v in d.items() if v is not None}

    def check(self, got, want=None, tokens=True):
        w = self.want() if want is None else want
        eq = lambda a, b, what: np.testing.assert_array_equal(a, np.asarray(b), err_msg=what)  # noqa: E731
        eq(got["status"], w["status"], "status")
        eq(got["bt"], w["block_tables"], "block tables")
        eq(got["kv_out"], w["kv_lens"], "lengths")
        eq(got["cu"], w["cu"], "prefix sums")
        eq(got["run"], w["run_request"], "runs")
        eq(got["slot0"], w["run_first_slot"], "first slots")
        if self.pages:
            eq(got["held_out"], w["n_blocks"], "blocks")
            eq(got["head_out"], [w["free_head"]], "head")
        if self.masks:
            eq(got["bp"], w["block_positions"], "block positions")
            eq(got["bm"].view(np.uint32), w["block_valid_mask"], "mask")
        if tokens:
            for name in ("slots", "positions", "requests"):
                full = np.full(self.room, -99, np.int64)
                for t, v in w[name].items():
                    full[t] = v
                eq(got[name], full, name)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("masks,offsets", [(False, False), (True, True)])
@pytest.mark.parametrize("P", [16, 32, 1, 7])
@pytest.mark.parametrize("B,new_hi", [(1, 1), (1, 3000), (3, 40), (64, 26), (65, 1), (272, 300), (1025, 9), (2500, 3)])
def test_tables_of_a_step(mepic, B, new_hi, P, masks, offsets, in_place):
    s = Step(B * 7 + P, B, P, new_hi=new_hi, masks=masks, offsets=offsets)
    want = s.want()
    s.check(s.run(mepic, in_place=in_place), want)


@pytest.mark.gpu
@pytest.mark.parametrize("B,new_hi", [(5, 40), (64, 26), (1500, 30)])
def test_a_list_that_runs_out(mepic, B, new_hi):
    """The first request that finds too few pages gets nothing, nor does any later one that needs some."""
    for short in (6, 7, 15, 10 ** 6):
        s = Step(B + short, B, 16, new_hi=new_hi, short=short, masks=True, head=3)
        want = s.want()
        assert 2 in want["status"] or short < 7
        s.check(s.run(mepic), want)


@pytest.mark.gpu
def test_tables_that_are_too_narrow_and_lengths_that_make_no_sense(mepic):
    s = Step(3, 300, 16, new_hi=60, width=12, masks=True)
    s.held = np.minimum(s.held, 12).astype(np.int32)
    s.kv = np.minimum(s.kv, 12 * 16).astype(np.int32)
    s.new[[7, 100]], s.kv[[30, 200]], s.new[250] = -3, -1, 2 ** 31 - 1
    s.room = 4000
    s.offsets = None
    want = s.want()
    assert {0, 1, 3} <= set(want["status"])
    got = s.run(mepic)
    total = int(np.clip(np.asarray(want["cu"], np.int64), 0, 2 ** 31 - 1)[-1])
    want["cu"] = np.clip(np.asarray(want["cu"], np.int64), 0, 2 ** 31 - 1)
    assert total == 2 ** 31 - 1
    s.check(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("pages", [False, True])
def test_without_token_arrays_and_without_a_list(mepic, pages):
    s = Step(8, 70, 16, new_hi=90, pages=pages, first=False)
    s.check(s.run(mepic, tokens=False), tokens=False)
    s.check(s.run(mepic))


@pytest.mark.gpu
def test_no_requests_and_no_tokens(mepic):
    s = Step(9, 0, 16, new_hi=5)
    s.check(s.run(mepic))
    s = Step(10, 12, 16, new_hi=0, masks=True)
    s.check(s.run(mepic))


@pytest.mark.gpu
def test_token_arrays_that_are_too_short(mepic):
    s = Step(11, 40, 16, new_hi=30, masks=True)
    s.room = s.room // 2
    s.check(s.run(mepic))


@pytest.mark.gpu
def test_page_ids_that_are_out_of_range_have_no_slots(mepic):
    s = Step(12, 20, 16, new_hi=30)
    s.bt[::3] = -4
    s.free[::2] = s.num_pages + 5
    s.check(s.run(mepic))


@pytest.mark.gpu
def test_captured_in_place_and_replayed(mepic):
    """A graph that grows the same requests again and again, from lengths the host never sees."""
    s = Step(13, 33, 16, new_hi=20, width=40, held_hi=5, spare=400, masks=True)
    got = s.run(mepic, in_place=True)
    want = s.want()
    s.check(got, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mepic.tables_extend(s.params)
    for _ in range(4):
        g.replay()
        torch.cuda.synchronize()
        s.bt, s.kv, s.held, s.head = want["block_tables"].astype(np.int32), np.array(want["kv_lens"], np.int32), np.array(want["n_blocks"], np.int32), want["free_head"]
        s.bp, s.bm = want["block_positions"].astype(np.int32), want["block_valid_mask"]
        want = s.want()
        s.check({k: v.cpu().numpy() for k, v in s.d.items() if v is not None}, want)


@pytest.mark.gpu
def test_runs_on_its_stream(mepic):
    s = Step(14, 33, 16, new_hi=20)
    s.run(mepic)
    new = s.d["new"].clone()
    s.d["new"].zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        s.d["new"].copy_(new)
    mepic.tables_extend(s.params, stream=side)
    side.synchronize()
    s.check({k: v.cpu().numpy() for k, v in s.d.items() if v is not None})


# ------------------------------------------------------------------------------------------------ refusals (no GPU)
def params(M, **over):
    p = M.ExtendParams()
    here = 1 << 20                                           # never dereferenced on the host
    base = dict(kv_lens=here, new_lens=here, block_tables=here, kv_lens_out=here, cu_tokens=here, run_request=here, run_first_slot=here, status=here,
                B=4, max_blocks=8, P=16, num_pages=100, workspace=here, workspace_bytes=1 << 20)
    base.update(over)
    for k, v in base.items():
        setattr(p, k, v)
    return p


def test_refusals_before_any_launch(mepic):
    lib = mepic.load()
    call = lambda **o: lib.mepic_tables_extend(ctypes.byref(params(mepic, **o)), None)  # noqa: E731
    here = 1 << 20
    for bad in (dict(kv_lens=None), dict(new_lens=None), dict(block_tables=None), dict(kv_lens_out=None), dict(cu_tokens=None), dict(run_request=None),
                dict(run_first_slot=None), dict(status=None), dict(B=-1), dict(max_blocks=-1), dict(P=0), dict(P=33), dict(num_pages=-1),
                dict(max_tokens=-1), dict(n_free=-1), dict(n_blocks=here), dict(n_blocks=here, n_blocks_out=here, free_head=here),
                dict(free_pages=here), dict(n_free=3), dict(n_blocks=here, n_blocks_out=here, free_head=here, free_head_out=here, n_free=3),
                dict(workspace=here + 8)):
        assert call(**bad) == mepic.ERR_INVALID, bad
    assert call(workspace=None) == mepic.ERR_CAPACITY and call(workspace_bytes=4) == mepic.ERR_CAPACITY
    assert lib.mepic_tables_extend(None, None) == mepic.ERR_INVALID
    assert lib.mepic_tables_extend_workspace_size(ctypes.byref(params(mepic)), None) == mepic.ERR_INVALID
    with pytest.raises(mepic.MepicError) as e:
        mepic.tables_extend_workspace_size(params(mepic, P=40))
    assert e.value.status == mepic.ERR_INVALID
    assert mepic.tables_extend_workspace_size(params(mepic)) > 0


def test_the_binding_looks_at_types_and_shapes(mepic):
    z = lambda *n, dt=torch.int32: torch.zeros(n, dtype=dt)  # noqa: E731
    good = dict(P=16, num_pages=9, kv_lens_out=z(3), cu_tokens=z(4), run_request=z(3), run_first_slot=z(3), status=z(3))
    for bad in (dict(cu_tokens=z(3)), dict(status=z(4)), dict(run_request=z(3, dt=torch.int64)), dict(token_slots=z(5)), dict(free_head=z(2)),
                dict(first_positions=z(2)), dict(token_positions=z(5), max_tokens=6), dict(block_positions=z(3, 4)),
                dict(block_valid_mask=z(3, 5, dt=torch.int64), max_tokens=0)):
        with pytest.raises(ValueError):
            mepic.make_extend_params(z(3), z(3), z(3, 5), **{**good, **bad})
    with pytest.raises(ValueError):
        mepic.make_extend_params(z(3), z(2), z(3, 5), **good)
