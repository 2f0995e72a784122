"""Embeddings, the router and rows in 8 bits without a GPU: what the C entries and the binding refuse, and sizes of workspaces."""
import ctypes as C

import pytest

from paper_2506_22668_amd import binding
from paper_2506_22668_amd.binding import DS_ECAPACITY, DS_EINVAL, DistShapError, Packed
from tests.test_feature_calls import P, _context, ctx  # noqa: F401

torch = pytest.importorskip("torch")

EMBED = dict(dtype=1, table_dtype=0, rows=5, cols=8, vocab=7, table=P, ts=8, ids=P, scale=1.0, y=P, ys=8)
EMBED_BACKWARD = dict(dtype=1, table_dtype=0, rows=100_000, cols=8, vocab=7, dy=P, dys=8, ids=P, scale=1.0, dtable=P, dts=8, ws=P, wsn=1 << 30)
ROUTE = dict(dtype=1, rows=100_000, experts=9, k=2, renorm=0, x=P, xs=9, ids=P, weights=P, counts=P, loss=P, lse=None, ws=P, wsn=1 << 20)
ROUTE_BACKWARD = dict(dtype=1, rows=5, experts=9, k=2, renorm=1, x=P, xs=9, lse=P, ids=P, counts=P, dweights=P, dloss=P, dx=P, dxs=9)
PACK = dict(dtype=0, rows=5, cols=40, x=P, xs=40, codes=P, cs=40, scales=P, ss=2)
UNPACK = dict(dtype=0, rows=5, cols=40, codes=P, cs=40, scales=P, ss=2, y=P, ys=40)
PACKED_BACKWARD = dict(dtype=1, rows=100_000, inner=40, outer=8, groups=3, dy=P, dys=8, codes=P, cs=40, scales=P, ss=2, w=P, offsets=P, order=None, gate=P, gs=40,
                       dx=P, dxs=40, dw=P, db=P, ws=P, wsn=1 << 40)
MANY = (1 << 30) + 1
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("name, good, bad", [
    ("ds_embed", EMBED, [dict(dtype=3), dict(table_dtype=2), dict(table_dtype=-1), dict(dtype=0, table_dtype=1), dict(rows=-1), dict(rows=MANY), dict(cols=0),
                         dict(cols=(1 << 20) + 1), dict(vocab=0), dict(vocab=MANY), dict(table=None), dict(table=P + 2), dict(ts=-1), dict(ids=None),
                         dict(scale=NAN), dict(scale=INF), dict(y=None), dict(y=P + 1), dict(ys=7)]),
    ("ds_embed_backward", EMBED_BACKWARD, [dict(dtype=3), dict(table_dtype=2), dict(rows=-1), dict(rows=MANY), dict(cols=0), dict(vocab=0), dict(vocab=MANY),
                                           dict(dy=None), dict(dy=P + 1), dict(ids=None), dict(scale=-INF), dict(dtable=None), dict(dtable=P + 2), dict(dts=7),
                                           dict(ws=P + 8)]),
    ("ds_route", ROUTE, [dict(dtype=3), dict(rows=-1), dict(rows=MANY), dict(experts=0), dict(experts=1025), dict(k=0), dict(k=9), dict(k=10), dict(experts=1, k=2),
                         dict(x=None), dict(x=P + 1), dict(xs=-9), dict(ids=None), dict(weights=None), dict(counts=None), dict(loss=None), dict(ws=P + 4)]),
    ("ds_route_backward", ROUTE_BACKWARD, [dict(dtype=3), dict(rows=-1), dict(experts=0), dict(experts=1025), dict(k=0), dict(k=9), dict(x=None), dict(lse=None),
                                           dict(ids=None), dict(counts=None), dict(dweights=None, dloss=None), dict(dx=None), dict(dxs=8)]),
    ("ds_pack_rows", PACK, [dict(dtype=3), dict(rows=-1), dict(cols=0), dict(cols=(1 << 20) + 1), dict(x=None), dict(x=P + 2), dict(codes=None), dict(cs=39),
                            dict(scales=None), dict(ss=1), dict(cs=-40), dict(cs=1 << 50)]),
    ("ds_unpack_rows", UNPACK, [dict(dtype=3), dict(rows=-1), dict(cols=0), dict(codes=None), dict(cs=-1), dict(scales=None), dict(ss=-1), dict(y=None),
                                dict(y=P + 1), dict(ys=39)]),
    ("ds_grouped_mm_backward_packed", PACKED_BACKWARD, [dict(dtype=3), dict(rows=-1), dict(rows=MANY), dict(inner=0), dict(outer=0), dict(groups=0),
                                                        dict(groups=1025), dict(dy=None), dict(codes=None), dict(cs=-1), dict(scales=None), dict(ss=-1), dict(w=None),
                                                        dict(offsets=None), dict(gs=-1), dict(dx=None), dict(dxs=39), dict(dw=None), dict(db=None), dict(ws=P + 2)]),
])
def test_bad_arguments_are_refused_before_any_work(ctx, name, good, bad):  # noqa: F811
    lib = binding.load_library()
    fn = getattr(lib, name)
    assert fn(None, *good.values()) == DS_EINVAL
    for change in bad:
        assert set(change) <= set(good)
        assert fn(ctx, *{**good, **change}.values()) == DS_EINVAL, change
        assert lib.ds_last_error(ctx), change


@pytest.mark.parametrize("name, good, sizes", [
    ("ds_embed_backward", EMBED_BACKWARD, (100_000, 8, 7)), ("ds_route", ROUTE, (100_000, 9)),
])
def test_a_workspace_that_is_too_small_is_refused(ctx, name, good, sizes):  # noqa: F811
    lib = binding.load_library()
    need = C.c_int64()
    assert getattr(lib, name + "_workspace")(*sizes, C.byref(need)) == 0 and need.value > 0
    for change in (dict(wsn=need.value - 1), dict(ws=None)):
        assert getattr(lib, name)(ctx, *{**good, **change}.values()) == DS_ECAPACITY


def test_a_workspace_of_packed_gradients_that_is_too_small_is_refused(ctx):  # noqa: F811
    lib = binding.load_library()
    need = C.c_int64()
    big = dict(rows=100_000, inner=512, outer=512, cs=512, ss=16, gs=512, dys=512, dxs=512)
    assert lib.ds_grouped_mm_backward_packed_workspace(1, 100_000, 512, 512, 3, C.byref(need)) == 0 and need.value > 0
    for change in (dict(wsn=need.value - 1), dict(ws=None)):
        assert lib.ds_grouped_mm_backward_packed(ctx, *{**PACKED_BACKWARD, **big, **change}.values()) == DS_ECAPACITY


def test_sizes_out_of_range_have_no_workspace():
    lib = binding.load_library()
    need = C.c_int64()
    for args in [(-1, 8, 8), (MANY, 8, 8), (8, 0, 8), (8, (1 << 20) + 1, 8), (8, 8, 0), (8, 8, MANY)]:
        assert lib.ds_embed_backward_workspace(*args, C.byref(need)) == DS_EINVAL
    for args in [(-1, 8), (MANY, 8), (8, 0), (8, 1025)]:
        assert lib.ds_route_workspace(*args, C.byref(need)) == DS_EINVAL
    for args in [(5, 1, 1, 1, 1), (0, -1, 1, 1, 1), (0, 1, 0, 1, 1), (0, 1, 1, 0, 1), (0, 1, 1, 1, 0)]:
        assert lib.ds_grouped_mm_backward_packed_workspace(*args, C.byref(need)) == DS_EINVAL
    assert lib.ds_embed_backward_workspace(8, 8, 8, None) == lib.ds_route_workspace(8, 8, None) == DS_EINVAL
    # the largest that are allowed have one
    assert lib.ds_embed_backward_workspace(1 << 30, 1 << 20, 1 << 30, C.byref(need)) == 0 and need.value > 1 << 40
    assert lib.ds_route_workspace(1 << 30, 1024, C.byref(need)) == 0 and need.value > 0


F32, BF16, I32, I64, U8, E4M3 = torch.float32, torch.bfloat16, torch.int32, torch.int64, torch.uint8, torch.float8_e4m3fn


def _held(rows=4, cols=40):
    return Packed(torch.zeros(rows, cols, dtype=U8).view(E4M3), torch.zeros(rows, (cols + 31) // 32, dtype=U8))


def _z(*shape, t=F32):
    return torch.zeros(*shape, dtype=t)


@pytest.mark.parametrize("call", [
    lambda c: c.embed(_z(4), _z(3, t=I32)),                                # not rows
    lambda c: c.embed(_z(4, 4, t=torch.float64), _z(3, t=I32)),
    lambda c: c.embed(_z(4, 4), _z(3, t=I64)),                             # ids are int32
    lambda c: c.embed(_z(4, 4), _z(3, 1, t=I32)),
    lambda c: c.embed(_z(4, 4), None),
    lambda c: c.embed(_z(4, 4), _z(3, t=I32), dtype=torch.float64),
    lambda c: c.embed_backward(_z(4), _z(4, t=I32), 5),
    lambda c: c.embed_backward(_z(4, 4), _z(3, t=I32), 5),                 # an id for every row
    lambda c: c.embed_backward(_z(4, 4), _z(4, t=I64), 5),
    lambda c: c.embed_backward(_z(4, 4), _z(4, t=I32), 5, dtype=torch.int32),
    lambda c: c.route(_z(4)),
    lambda c: c.route(_z(4, 4, t=torch.float64)),
    lambda c: c.route_backward(_z(4, 4), _z(4), _z(2, 4, t=I64), _z(5, t=I64), dweights=_z(2, 4)),
    lambda c: c.route_backward(_z(4, 4), _z(4), _z(2, 3, t=I32), _z(5, t=I64), dweights=_z(2, 4)),
    lambda c: c.route_backward(_z(4, 4), _z(3), _z(2, 4, t=I32), _z(5, t=I64), dweights=_z(2, 4)),
    lambda c: c.route_backward(_z(4, 4), _z(4), _z(2, 4, t=I32), _z(4, t=I64), dweights=_z(2, 4)),
    lambda c: c.route_backward(_z(4, 4), _z(4), _z(2, 4, t=I32), _z(5, t=I64), dweights=_z(1, 4)),
    lambda c: c.route_backward(_z(4, 4), _z(4), _z(2, 4, t=I32), _z(5, t=I64), dloss=_z(2)),
    lambda c: c.route_backward(_z(4, 4), None, _z(2, 4, t=I32), _z(5, t=I64), dloss=_z(1)),
    lambda c: c.pack_rows(_z(4)),
    lambda c: c.pack_rows(_z(4, 4, t=torch.float64)),
    lambda c: c.unpack_rows(_z(4, 4)),                                     # not packed
    lambda c: c.unpack_rows(_held(), torch.float64),
    lambda c: c.unpack_rows(Packed(_z(4, 40, t=U8), _z(4, 2, t=U8))),      # codes are e4m3
    lambda c: c.unpack_rows(Packed(_held().codes, _z(4, 2))),
    lambda c: c.unpack_rows(Packed(_held().codes, _z(4, 1, t=U8))),        # a scale for every block
    lambda c: c.grouped_mm_backward(_z(4, 8), _held(), _z(2, 41, 8), _z(3, t=I64)),
    lambda c: c.grouped_mm_backward(_z(4, 8), _held(), _z(2, 40, 8), _z(2, t=I64)),
    lambda c: c.grouped_mm_backward(_z(4, 8), _held(), _z(2, 40, 8), None),
    lambda c: c.grouped_mm_backward(_z(4, 8), _held(), _z(2, 40, 8, t=torch.float64), _z(3, t=I64)),
    lambda c: c.grouped_mm_backward(_z(4, 8, t=BF16), _held(), _z(2, 40, 8), _z(3, t=I64)),
    lambda c: c.grouped_mm_backward(_z(3, 8), _held(), _z(2, 40, 8), _z(3, t=I64)),
    lambda c: c.grouped_mm_backward(_z(4, 8), _held(), _z(2, 40, 8), _z(3, t=I64), order=_z(4, t=I64)),
    lambda c: c.grouped_mm_backward(_z(4, 8), _held(), _z(2, 40, 8), _z(3, t=I64), gate=_z(4, 40)),      # a gate that is not packed
    lambda c: c.grouped_mm_backward(_z(4, 8), _held(), _z(2, 40, 8), _z(3, t=I64), gate=_held(4, 41)),
    lambda c: c.grouped_mm_backward(_z(4, 8), _z(4, 40), _z(2, 40, 8), _z(3, t=I64), gate=_held()),      # a packed gate of rows that are not
])
def test_the_binding_refuses_shapes_and_types(call):
    with pytest.raises(DistShapError) as e:
        call(_context())
    assert e.value.code == DS_EINVAL


def test_tensors_of_another_device_are_refused():
    c = _context()
    c._index, c.device = 0, torch.device("cuda:0")
    for call in (lambda: c.embed(_z(4, 4), _z(3, t=I32)), lambda: c.route(_z(4, 4)), lambda: c.pack_rows(_z(4, 4)), lambda: c.unpack_rows(_held()),
                 lambda: c.grouped_mm_backward(_z(4, 8), _held(), _z(2, 40, 8), _z(3, t=I64))):
        with pytest.raises(DistShapError):
            call()


@pytest.mark.parametrize("k", [0, -1, 5, 9])
def test_more_experts_than_there_are_are_refused(k):
    c = _context()
    c.lib = binding.load_library()
    with pytest.raises(DistShapError):
        c.route(_z(4, 4), k)
