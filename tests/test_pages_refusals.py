"""What the paged cache's calls refuse, before anything is launched: no GPU."""
import ctypes as C

import pytest
import torch

import paper_2502_00937_amd as V
from paper_2502_00937_amd import pages as P

FAKE = 1 << 20  # a pointer that nothing reads: every call below is refused on the host or has nothing to do


def plan(lib, **kw):
    a = dict(cached=FAKE, new=FAKE, table=FAKE, free=FAKE, taken=0, slots=FAKE, offsets=FAKE, kv=FAKE, firsts=FAKE, counts=FAKE, stride=8,
             n=4, width=8, n_free=9, n_pages=16, page=16, rows=10)
    assert set(kw) <= set(a)
    return lib.vit_pages_plan(P._PLAN.pack(*dict(a, **kw).values()), None)


def append(lib, **kw):
    a = dict(k=FAKE, v=FAKE, slots=FAKE, kp=FAKE, vp=FAKE, k_stride=256, v_stride=256, rows=4, n_pages=16, page=16, heads=2, dim=64, dtype=1)
    assert set(kw) <= set(a)
    return lib.vit_pages_append(P._APPEND.pack(*dict(a, **kw).values()), None)


ATTEND = dict(q=FAKE, kp=FAKE, vp=FAKE, table=FAKE, offsets=FAKE, kv=FAKE, out=FAKE, ws=0, ws_bytes=0, q_stride=512, out_stride=512,
              table_stride=8, rows=4, n=2, max_new=4, width=8, n_pages=16, page=16, heads=8, kv_heads=2, dim=64, causal=1, dtype=1, scale=0.125)


def attend(lib, **kw):
    assert set(kw) <= set(ATTEND)
    return lib.vit_pages_attend(P._ATTEND.pack(*dict(ATTEND, **kw).values()), None)


def test_plan_refuses():
    lib = V.load_library()
    assert lib.vit_pages_plan(None, None) == -1
    for bad in ({"n": -1}, {"n": (1 << 20) + 1}, {"width": -1}, {"width": 9}, {"n_free": -1}, {"rows": -1}, {"rows": 1 << 30},
                {"page": 0}, {"page": 4}, {"page": 24}, {"page": 8192}, {"n_pages": -1}, {"n_pages": 1 << 27}):
        assert plan(lib, **bad) == -1, bad
    for name in ("cached", "new", "table", "free", "slots", "offsets", "kv", "firsts", "counts"):
        assert plan(lib, **{name: 0}) == -1, name
        assert b"NULL" in lib.vit_last_error()


def test_append_refuses():
    lib = V.load_library()
    assert lib.vit_pages_append(None, None) == -1
    for bad in ({"rows": -1}, {"k_stride": 127}, {"v_stride": 127}, {"k_stride": 1 << 33}, {"page": 12}, {"n_pages": -1}, {"n_pages": 1 << 27},
                {"heads": 0}, {"heads": 1025}, {"dim": 0}, {"dim": 12}, {"dim": 136}, {"dtype": 2}, {"k": FAKE + 8}, {"vp": FAKE + 4},
                {"k_stride": 260}, {"v_stride": 257}):
        assert append(lib, **bad) == -1, bad
    for name in ("k", "v", "slots", "kp", "vp"):
        assert append(lib, **{name: 0}) == -1, name
    assert append(lib, rows=0, k=0, v=0, slots=0) == 0  # nothing to do


def test_attend_refuses():
    lib = V.load_library()
    assert lib.vit_pages_attend(None, None) == -1
    for bad in ({"rows": -1}, {"rows": 1 << 30}, {"n": -1}, {"n": (1 << 20) + 1}, {"max_new": -1}, {"width": -1}, {"width": 9}, {"n_pages": -1},
                {"n_pages": 1 << 27}, {"page": 7}, {"heads": 9}, {"heads": 0}, {"heads": 1026}, {"kv_heads": 0}, {"dim": 60}, {"dim": 192},
                {"dtype": -1}, {"scale": float("nan")}, {"scale": float("inf")}, {"q_stride": 511}, {"out_stride": 504}, {"q_stride": 514},
                {"out_stride": 1 << 33}, {"q": FAKE + 8}, {"out": FAKE + 2}, {"kp": FAKE + 4}, {"ws": FAKE + 16}):
        assert attend(lib, **bad) == -1, bad
    for name in ("q", "kp", "vp", "table", "offsets", "kv", "out"):
        assert attend(lib, **{name: 0}) == -1, name
    assert attend(lib, rows=0) == 0 and attend(lib, n=0) == 0 and attend(lib, max_new=0) == 0  # nothing to do
    need = C.c_size_t(123)
    assert lib.vit_pages_attend_query(None, C.byref(need)) == -1
    assert lib.vit_pages_attend_query(P._ATTEND.pack(*ATTEND.values()), None) == -1
    assert lib.vit_pages_attend_query(P._ATTEND.pack(*dict(ATTEND, dim=60).values()), C.byref(need)) == -1 and need.value == 123
    assert lib.vit_pages_attend_query(P._ATTEND.pack(*ATTEND.values()), C.byref(need)) == 0
    if need.value:  # a workspace that is missing or one byte short
        assert attend(lib) == -3 and attend(lib, ws=FAKE, ws_bytes=need.value - 1) == -3


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def refused(call, *args, **kw):
    with pytest.raises(V.VitError) as e:
        call(*args, **kw)
    assert e.value.status == V.binding.VIT_EINVAL
    return str(e.value)


def test_binding_refuses_tensors_that_do_not_fit():
    pool = torch.zeros(6, 2, 16, 64, dtype=torch.bfloat16)
    rows = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    # right in everything but the place: there is no path on the CPU
    assert "on a GPU" in refused(V.append_pages, rows, rows, ints(5), pool, pool)
    assert "on a GPU" in refused(V.plan_pages, ints(2), ints(2), ints(2, 4), ints(3), None, 6, 16, 7)
    assert "on a GPU" in refused(V.plan_pages, ints(2), ints(2), ints(2, 9)[:, :4], ints(3), ints(1), 6, 16, 7)
    good = dict(q=torch.zeros(5, 4, 64, dtype=torch.bfloat16), key_pages=pool, value_pages=pool, block_table=ints(2, 4), query_offsets=ints(3),
                kv_lens=ints(2), max_new=3)
    assert "on a GPU" in refused(V.attend_pages, **good)
    assert "on a GPU" in refused(V.attend_pages, **dict(good, q=torch.zeros(5, 8, 64, dtype=torch.bfloat16)[:, :4]))
    for name, bad in (("key_pages", pool.half()), ("key_pages", pool[0]), ("key_pages", pool.transpose(1, 2)), ("value_pages", pool.float()),
                      ("value_pages", pool[:5]), ("q", good["q"].float()), ("q", good["q"][:, :, :32]), ("q", good["q"].transpose(0, 1).contiguous().transpose(0, 1)),
                      ("q", good["q"][0]), ("block_table", ints(2, 4).long()), ("block_table", ints(4, 2).t()), ("block_table", ints(8)),
                      ("block_table", ints(3, 4)), ("query_offsets", ints(2)), ("kv_lens", ints(3)), ("kv_lens", ints(4)[::2]), ("out", good["q"][:4]),
                      ("out", good["q"].float())):
        assert "on a GPU" not in refused(V.attend_pages, **dict(good, **{name: bad})), (name, bad.shape)
    for args in ((rows[:4], rows, ints(5)), (rows, rows[:4], ints(5)), (rows, rows, ints(4)), (rows, rows.float(), ints(5)),
                 (rows[:, :1], rows, ints(5)), (rows, rows, ints(5).long()), (rows, rows, ints(10)[::2])):
        assert "on a GPU" not in refused(V.append_pages, *args, pool, pool)
    for args in ((ints(3), ints(2), ints(2, 4), ints(3), None), (ints(2), ints(1), ints(2, 4), ints(3), None), (ints(2), ints(2), ints(2, 4).long(), ints(3), None),
                 (ints(2), ints(2), ints(2, 4), ints(3).float(), None), (ints(2), ints(2), ints(2, 4), ints(3), ints(0)), (ints(2), ints(2), ints(4, 2).t(), ints(3), None)):
        assert "on a GPU" not in refused(V.plan_pages, *args, 6, 16, 7)
    refused(V.plan_pages, ints(2), ints(2), ints(2, 4), ints(3), None, 6, 16, -1)
    wrong = V.PagePlan(ints(7), ints(3), ints(2), ints(3), ints(1))
    assert "counts" in refused(V.plan_pages, ints(2), ints(2), ints(2, 4), ints(3), None, 6, 16, 7, out=wrong)


def test_launches_that_have_no_room_are_refused():
    """More threads than a launch has (2^32): an error ahead of the launch, not one of it."""
    lib = V.load_library()
    assert append(lib, rows=1 << 23, heads=32, dim=128, k_stride=4096, v_stride=4096) == -1
    assert b"64 GiB" in lib.vit_last_error()
    assert attend(lib, rows=1 << 26, n=1 << 20, max_new=1 << 10, heads=16, kv_heads=16, q_stride=1024, out_stride=1024) == -1
    assert b"workgroups" in lib.vit_last_error()


@pytest.mark.parametrize("number", [2 ** 31, -2 ** 31 - 1, 2 ** 70, 1.5])
def test_binding_refuses_numbers_that_no_field_holds(number):
    pool = torch.zeros(6, 2, 16, 64, dtype=torch.bfloat16)
    q = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    assert "range" in refused(V.attend_pages, q, pool, pool, ints(2, 4), ints(3), ints(2), number)
    assert "range" in refused(V.plan_pages, ints(2), ints(2), ints(2, 4), ints(3), None, number, 16, 7)
    assert "range" in refused(V.plan_pages, ints(2), ints(2), ints(2, 4), ints(3), None, 6, number, 7)
    assert "scale" in refused(V.attend_pages, q, pool, pool, ints(2, 4), ints(3), ints(2), 3, scale=1e39)  # (infinite as a float)


def test_structs_match_the_header():
    """The packed formats follow include/vitenc.h: field sizes in order."""
    import os
    import re

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "vitenc.h")).read(), flags=re.S)
    for name, packed in (("plan", P._PLAN), ("append", P._APPEND), ("attend", P._ATTEND)):
        body = re.findall(r"typedef struct \{([^}]*)\} vit_pages_%s_t;" % name, text)[0]
        codes = ""
        for kind, star in re.findall(r"(?:const )?(\w+)\s*(\*?)\s*\w+;", body):
            codes += "Q" if star or kind == "size_t" else {"int64_t": "q", "int32_t": "i", "float": "f"}[kind]
        assert codes == re.sub(r"(\d+)(\w)", lambda m: m[2] * int(m[1]), packed.format)
