"""CPU-only checks of the router's, the exchange's and the clipping's C entries: symbols, struct layouts, refusals before
anything touches a GPU, and the clipping's table, which is made on the host."""
import ctypes as C
import math
import os
import random
import re
import subprocess

import pytest

from paper_1901_01544_b200 import binding, build, clipping, routing

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E = binding.IWP_ERR_INVALID
HEADERS = {"iwp_route.h": routing, "iwp_clip.h": clipping}


@pytest.fixture(scope="module")
def L():
    build.build()
    routing.lib()
    return clipping.lib()


@pytest.mark.parametrize("name", HEADERS)
def test_header_and_library_agree(L, name):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", name)).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(iwp_[a-z_0-9]+)\s*\(", src)))
    assert names == sorted(HEADERS[name].EXPORTS)
    for n in names:
        assert hasattr(L, n)


def test_structs_have_the_headers_layout(tmp_path):
    fields = {"iwp_route_args": routing.RouteArgs, "iwp_route_grad_args": routing.RouteGradArgs, "iwp_order_args": routing.OrderArgs,
              "iwp_exchange_args": routing.ExchangeArgs, "iwp_clip_args": clipping.ClipArgs, "iwp_clip_tensor": clipping.ClipTensor,
              "iwp_clip_sizes": clipping.ClipSizes}
    lines = ['#include "%s"' % os.path.join(ROOT, "include", h) for h in HEADERS] + ["#include <cstddef>", "#include <cstdio>", "int main() {"]
    for name, cls in fields.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        for f, _ in cls._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, f.rstrip("_")))
    lines.append('printf("%d\\n", IWP_ROUTE_STATE);')
    (tmp_path / "l.cpp").write_text("\n".join(lines + ["}"]))
    subprocess.run(["g++", str(tmp_path / "l.cpp"), "-o", str(tmp_path / "l")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for cls in fields.values():
        want += [C.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want + [routing.ROUTE_STATE]


def made(cls, base, kw):
    a = cls(**base)
    for k, v in kw.items():
        setattr(a, k, v)
    return C.byref(a)


ROUTE = dict(tokens=8, experts=16, top_k=2, groups=1, top_groups=1, group_top=2, type=0, ids_bytes=4, logits=256, logits_ld=16, ids=256, weights=256,
             counts=256, state=256, weight_scale=1.0)
GRAD = dict(tokens=8, experts=16, top_k=2, type=0, ids_bytes=4, logits=256, logits_ld=16, ids=256, ids_ld=2, weights=256, weights_ld=2, dweights=256,
            dweights_ld=2, dlogits=256, dlogits_ld=16, weight_scale=1.0, scale=1.0)
ORDER = dict(tokens=8, experts=16, top_k=2, ids_bytes=4, ids=256, ids_ld=2, offsets=256, slots=256, rows=256, workspace=256, workspace_bytes=1 << 30)
ROWS = dict(tokens=8, dim=16, experts=16, top_k=2, type=0, slots=256, offsets=256, by_token=256, by_token_ld=16, by_slot=256, by_slot_ld=16, weights=256,
            weights_ld=2, by_token_out=256, by_token_out_ld=16, by_slot_out=256, by_slot_out_ld=16, dweights=256)
CLIP = dict(table=256, parts=1, warps=1, squares=256, norms=256, factors=256, workspace=256, workspace_bytes=1 << 20, state=256, max_norm=1.0, scale=1.0,
            groups=1, write=1)


@pytest.mark.parametrize("bad", [
    dict(tokens=-1), dict(tokens=1 << 31), dict(experts=0), dict(experts=1025), dict(top_k=0), dict(top_k=17), dict(experts=64, logits_ld=64, top_k=33),
    dict(groups=0), dict(groups=3), dict(groups=33), dict(groups=4, top_groups=0), dict(groups=4, top_groups=5), dict(groups=4, top_groups=1, top_k=5),
    dict(groups=16, top_groups=2), dict(group_top=0), dict(group_top=3), dict(score=2), dict(weight_scale=0.0), dict(weight_scale=math.inf),
    dict(type=3), dict(ids_bytes=2), dict(logits=None), dict(logits=258), dict(logits_ld=15), dict(ids=None), dict(ids=260, ids_bytes=8), dict(weights=None),
    dict(weights=258), dict(bias=257), dict(counts=258), dict(state=None), dict(state=128)])
def test_route_refuses(L, bad):
    assert L.iwp_route(made(routing.RouteArgs, ROUTE, bad), None) == E


@pytest.mark.parametrize("bad", [
    dict(tokens=-1), dict(experts=0), dict(top_k=0), dict(score=5), dict(weight_scale=0.0), dict(scale=math.nan), dict(type=-1), dict(ids_bytes=3),
    dict(logits=None), dict(ids=None), dict(weights=None), dict(dweights=None), dict(dlogits=None), dict(logits_ld=15), dict(ids_ld=1), dict(weights_ld=1),
    dict(dweights_ld=1), dict(dlogits_ld=15), dict(dlogits=258), dict(dweights=258), dict(dlogits_ld=1 << 40)])
def test_route_grad_refuses(L, bad):
    assert L.iwp_route_grad(made(routing.RouteGradArgs, GRAD, bad), None) == E


@pytest.mark.parametrize("bad", [
    dict(tokens=-1), dict(tokens=1 << 30), dict(experts=0), dict(experts=1025), dict(top_k=0), dict(top_k=33), dict(ids=None), dict(ids_ld=1), dict(ids_bytes=1),
    dict(offsets=None), dict(slots=None), dict(rows=None), dict(workspace=None), dict(workspace=128), dict(rows=257)])
def test_order_refuses(L, bad):
    assert L.iwp_order(made(routing.OrderArgs, ORDER, bad), None) == E


@pytest.mark.parametrize("entry,bad", [
    *[(e, b) for e in ("iwp_dispatch", "iwp_combine", "iwp_combine_grad") for b in (
        dict(tokens=-1), dict(tokens=1 << 30), dict(dim=0), dict(dim=1 << 31), dict(tokens=1 << 28, dim=1 << 20), dict(top_k=0), dict(top_k=33), dict(experts=0),
        dict(type=4), dict(slots=None), dict(offsets=None), dict(weights_ld=1), dict(weights=257))],
    ("iwp_dispatch", dict(by_token=None)), ("iwp_dispatch", dict(by_slot_out=None)), ("iwp_dispatch", dict(by_token_ld=15)), ("iwp_combine", dict(by_slot=None)),
    ("iwp_combine", dict(by_token_out=258)), ("iwp_combine", dict(by_slot_ld=15)), ("iwp_combine_grad", dict(by_slot=None)),
    ("iwp_combine_grad", dict(by_slot_out=None, dweights=None)), ("iwp_combine_grad", dict(by_slot_out_ld=15)), ("iwp_combine_grad", dict(dweights=258))])
def test_exchange_refuses(L, entry, bad):
    assert getattr(L, entry)(made(routing.ExchangeArgs, ROWS, bad), None) == E


@pytest.mark.parametrize("bad", [
    dict(table=None), dict(table=264), dict(parts=-1), dict(parts=1 << 27), dict(warps=-1), dict(warps=4737), dict(squares=None), dict(squares=260), dict(norms=None), dict(factors=None),
    dict(workspace=None), dict(workspace=128), dict(state=None), dict(state=64), dict(max_norm=-1.0), dict(max_norm=math.nan), dict(scale=0.0), dict(scale=math.inf),
    dict(groups=0), dict(groups=(1 << 20) + 1)])
def test_clip_refuses(L, bad):
    assert L.iwp_clip(made(clipping.ClipArgs, CLIP, bad), None) == E


def test_nothing_and_too_little(L):
    for entry in ("iwp_route", "iwp_route_grad", "iwp_order", "iwp_dispatch", "iwp_combine", "iwp_combine_grad", "iwp_clip"):
        assert getattr(L, entry)(None, None) == E
    assert L.iwp_route_reset(None, None) == E
    need = L.iwp_order_workspace(made(routing.OrderArgs, ORDER, {}))
    assert need > 0 and L.iwp_order_workspace(made(routing.OrderArgs, ORDER, dict(experts=0))) == -1 and L.iwp_order_workspace(None) == -1
    assert L.iwp_order(made(routing.OrderArgs, ORDER, dict(workspace_bytes=need - 1)), None) == binding.IWP_ERR_CAPACITY
    assert L.iwp_clip(made(clipping.ClipArgs, CLIP, dict(warps=300, workspace_bytes=8 * 301 - 1)), None) == binding.IWP_ERR_CAPACITY
    for entry in ("iwp_route_grad", "iwp_dispatch", "iwp_combine", "iwp_combine_grad"):  # no tokens: nothing to do, no launch
        cls, base = (routing.RouteGradArgs, GRAD) if entry == "iwp_route_grad" else (routing.ExchangeArgs, ROWS)
        assert getattr(L, entry)(made(cls, base, dict(tokens=0)), None) == binding.IWP_OK


# ---- the clipping's table -------------------------------------------------------------------------------


class Part(C.Structure):
    _fields_ = [("in_", C.c_uint64), ("out", C.c_uint64), ("in_ld", C.c_int64), ("out_ld", C.c_int64), ("rows", C.c_int32), ("cols", C.c_int32),
                ("group", C.c_int32), ("in_type", C.c_int16), ("out_type", C.c_int16)]


class Start(C.Structure):
    _fields_ = [("part", Part), ("next", C.c_int32), ("end", C.c_int32), ("fill", C.c_int32 * 2)]


def table_of(L, tensors, groups):
    """Parts of each warp, in order, and where each group's sums are."""
    arr = (clipping.ClipTensor * max(1, len(tensors)))(*tensors)
    sizes = clipping.ClipSizes()
    assert L.iwp_clip_layout(arr, len(tensors), groups, C.byref(sizes)) == binding.IWP_OK
    raw = (C.c_uint64 * (sizes.table_bytes // 8))()
    assert L.iwp_clip_table(arr, len(tensors), groups, raw, sizes.table_bytes - 1) == binding.IWP_ERR_CAPACITY
    assert L.iwp_clip_table(arr, len(tensors), groups, raw, sizes.table_bytes) == binding.IWP_OK
    at = C.addressof(raw)
    warps = sizes.warps
    starts = [Start.from_buffer_copy(s) for s in (Start * warps).from_address(at)] if warps else []
    at += warps * C.sizeof(Start)
    parts = [Part.from_buffer_copy(p) for p in (Part * sizes.parts).from_address(at)] if sizes.parts else []
    at += sizes.parts * C.sizeof(Part)
    spans = [tuple(s) for s in (C.c_int32 * 2 * groups).from_address(at)]
    assert at + 8 * groups <= C.addressof(raw) + sizes.table_bytes
    return sizes, [[s.part] + parts[s.next : s.end] if s.end >= 0 else [] for s in starts], spans, parts


@pytest.mark.parametrize("total", [0, 5, 5000, 300_000, 40_000_000])
def test_every_element_is_in_one_part_of_its_group(L, total):
    rng = random.Random(total)
    groups, tensors, at, left = 4, [], 1 << 20, total
    while left > 0:
        rows, cols = rng.choice([(1, rng.randint(1, 1 + left // 3)), (rng.randint(1, 50), rng.randint(1, 90)), (3, 20000)])
        ld = cols + rng.choice([0, 0, 5])
        tensors.append(clipping.ClipTensor(at, 2 * at, rows, cols, ld, ld, rng.choice([0, 1, 3]), rng.choice([0, 1, 2]), rng.choice([0, 1, 2])))
        at += rows * ld * 4 + 64
        left -= rows * cols
    sizes, warps, spans, listed = table_of(L, tensors, groups)
    elements = sum(t.rows * t.cols for t in tensors)
    assert sizes.workspace_bytes >= 8 * (len(warps) + groups)
    parts = [p for w in warps for p in w]
    assert bytes(b"".join(parts)) == bytes(b"".join(listed))
    # a warp's sum over a group has a place of its own, among the group's
    places = [(w + p.group, w, p.group) for w, mine in enumerate(warps) for p in mine]
    assert len({q[0] for q in places}) == len({q[1:] for q in places}) and max((q[0] for q in places), default=0) < len(warps) + groups
    for g in range(groups):
        own = {q[0] for q in places if q[2] == g}
        assert own == set(range(*spans[g])), (g, spans[g])
    cost = [sum(1024 + p.rows * p.cols for p in mine) for mine in warps]
    assert sum(cost) == elements + 1024 * len(parts)
    if warps:  # shared out evenly: what a range cut short leaves of it, and rounding
        assert max(cost) <= sizes.range <= 1.1 * sum(cost) / len(cost) + 2 * 1024 + 3 * 128
    if total > 1_000_000:  # (element by element below)
        return
    width = {0: 4, 1: 2, 2: 2}

    def elements(things):
        return sorted((t.in_ + (r * t.in_ld + c) * width[t.in_type], t.out + (r * t.out_ld + c) * width[t.out_type], t.group, t.in_type, t.out_type)
                      for t in things for r in range(t.rows) for c in range(t.cols))

    assert elements(parts) == elements(tensors)


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(cols=-1), dict(group=-1), dict(group=2), dict(in_type=3), dict(out_type=-1), dict(in_=None), dict(in_=258), dict(out=257), dict(cols=1 << 47),
    dict(rows=1 << 40, cols=1 << 40), dict(in_ld=-1), dict(out_ld=9)])
def test_table_refuses(L, bad):
    base = dict(in_=256, out=4096, rows=3, cols=10, in_ld=10, out_ld=10, group=0, in_type=0, out_type=0)
    t = clipping.ClipTensor(**(base | bad))
    sizes = clipping.ClipSizes()
    assert L.iwp_clip_layout(C.byref(t), 1, 2, C.byref(sizes)) == E
    good = clipping.ClipTensor(**base)
    assert L.iwp_clip_layout(C.byref(good), 1, 2, None) == E and L.iwp_clip_layout(None, 1, 2, C.byref(sizes)) == E
    assert L.iwp_clip_layout(C.byref(good), -1, 2, C.byref(sizes)) == E and L.iwp_clip_layout(C.byref(good), 1, 0, C.byref(sizes)) == E
    assert L.iwp_clip_table(C.byref(good), 1, 2, None, 1 << 20) == E


def test_strided_shapes_are_cut_into_runs():
    runs = clipping._runs
    assert runs((), ((), ())) == [((0, 0), 1, 1, (0, 0))]
    assert runs((4, 5, 6), ((30, 6, 1), (30, 6, 1))) == [((0, 0), 1, 120, (0, 0))]
    assert runs((4, 5), ((1, 4), (1, 4))) == [((0, 0), 1, 20, (0, 0))]
    assert runs((4, 5), ((10, 1), (5, 1))) == [((0, 0), 4, 5, (10, 5))]
    assert runs((2, 3, 4), ((100, 10, 1), (100, 20, 1))) == [((0, 0), 3, 4, (10, 20)), ((100, 100), 3, 4, (10, 20))]
    assert runs((7, 1, 3), ((0, 9, 1), (0, 9, 1))) == [((0, 0), 7, 3, (0, 0))]
    for shape, strides in (((4, 5), ((10, 2), (10, 2))), ((4, 5), ((1, 4), (5, 1)))):
        with pytest.raises(ValueError):
            runs(shape, strides)
