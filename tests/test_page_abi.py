"""The paged entries on the CPU: exports, refusals on the host before any device work, the reference's own layout.
(No compute call runs here: there is no GPU.)"""
import ctypes
import os
import re

import numpy as np
import pytest

import page_reference as ref
import paper_2605_30574_amd as sp
from paper_2605_30574_amd import pages as PG

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # never dereferenced: every call here is refused, or has nothing to do


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "splice_pages.h")).read()
    declared = set(re.findall(r"SPLICE_API\s+[\w\s\*]+?\b(splice_\w+)\s*\(", text))
    assert declared == set(PG.EXPORTS)
    lib = sp.load_library()
    for name in declared:
        assert hasattr(lib, name) and hasattr(sp, name), name


def shape(**kw):
    base = dict(n_cells=3, n_layers=4, n_q_heads=8, n_kv_heads=2, head_dim=64, prompt_len=32, span=(4, 28), gen_capacity=100,
                donor_zero=False, dtype="bf16")
    base.update(kw)
    return sp.make_shape(**base)


def ints(*x):
    return (ctypes.c_int32 * len(x))(*x)


STEPS, LW, NEW = ints(0, 5, -1), ints(0, 0, 1, 2, 9, 0), ints(4, 1, 0)


def attn(sh=None, pages=None, steps=STEPS, new=NEW, call=None, LW=LW, **kw):
    a = dict(tables=FAKE, clean=FAKE, donor=FAKE, q=FAKE, pool=FAKE, out=FAKE, lse=FAKE, ws=FAKE, bytes=1 << 40)
    a.update(kw)
    return PG._library().splice_page_attn(sh or shape(), call or sp.make_call(1, 0, 0, 0.125), pages or sp.make_pages(9, 2, 4), LW, steps,
                                          new, *a.values(), None)


def append(sh=None, pages=None, steps=STEPS, new=NEW, rope=None, **kw):
    a = dict(tables=FAKE, pos=None, freq=FAKE, q=FAKE, qs=512, k=FAKE, ks=128, v=FAKE, vs=128, q_out=2 * FAKE, pool=FAKE)
    a.update(kw)
    return PG._library().splice_page_append(sh or shape(), pages or sp.make_pages(9, 2, 4), rope or sp.make_rope("half", 64), steps, new,
                                            *a.values(), None)


def read(sh=None, pages=None, steps=STEPS, new=NEW, **kw):
    a = dict(tables=FAKE, pool=FAKE, rk=FAKE, rv=FAKE)
    a.update(kw)
    return PG._library().splice_page_read(sh or shape(), pages or sp.make_pages(9, 2, 4), steps, new, *a.values(), None)


def compact(sh=None, pages=None, steps=STEPS, **kw):
    a = dict(keep=FAKE, tables=FAKE, pool=FAKE, stride=9 * 2 * 68 * 64)
    a.update(kw)
    return PG._library().splice_page_compact(sh or shape(), pages or sp.make_pages(9, 2, 4), steps, *a.values(), None)


def fork(sh=None, pages=None, parent=ints(0, 0, -1), rows=ints(5, 5, 0), want=ints(9, 128, 0), **kw):
    a = dict(tables=FAKE, refs=FAKE, new_tables=2 * FAKE, new_refs=2 * FAKE, missing=FAKE, copied=FAKE, pool=FAKE,
             stride=9 * 2 * 68 * 64)
    a.update(kw)
    return PG._library().splice_page_fork(sh or shape(), pages or sp.make_pages(9, 2, 4), parent, rows, want, *a.values(), None)


@pytest.mark.parametrize("entry", [attn, append, read, compact, fork])
def test_shapes_and_pages(entry):
    assert entry(sh=shape(dtype="f32")) == sp.SPLICE_EUNSUPPORTED
    assert entry(sh=shape(head_dim=96)) == sp.SPLICE_EUNSUPPORTED
    assert entry(sh=shape(n_q_heads=6)) == sp.SPLICE_EUNSUPPORTED
    assert entry(sh=shape(n_q_heads=1 << 16, n_kv_heads=1 << 16)) == sp.SPLICE_EUNSUPPORTED
    assert entry(sh=shape(n_layers=1 << 16)) == sp.SPLICE_EUNSUPPORTED
    assert entry(sh=shape(n_cells=257)) == sp.SPLICE_EUNSUPPORTED
    assert entry(sh=shape(span=(4, 33))) == sp.SPLICE_ESHAPE
    assert entry(sh=shape(gen_capacity=129)) == sp.SPLICE_ESHAPE          # more rows than a table names
    for bad in (sp.make_pages(0, 2, 4), sp.make_pages(9, 0, 4), sp.make_pages(9, 2, 0)):
        assert entry(pages=bad) == sp.SPLICE_ESHAPE
    for much in (sp.make_pages((1 << 24) + 1, 2, 4), sp.make_pages(9, (1 << 22) + 1, 4), sp.make_pages(9, 2, 32769)):
        assert entry(pages=much) == sp.SPLICE_EUNSUPPORTED
    assert entry(pool=None) == sp.SPLICE_EINVAL
    assert entry(pool=FAKE + 8) == sp.SPLICE_EINVAL
    assert entry(tables=None) == sp.SPLICE_EINVAL
    assert entry(tables=FAKE + 2) == sp.SPLICE_EINVAL
    assert entry(sh=shape(n_cells=0)) == sp.SPLICE_OK


@pytest.mark.parametrize("entry", [attn, append, read])
def test_steps_and_tokens(entry):
    assert entry(steps=None) == sp.SPLICE_EINVAL
    assert entry(steps=ints(97, 0, -1)) == sp.SPLICE_ESHAPE               # 97 + 4 > 100
    assert entry(steps=ints(0, 2**31 - 1, -1)) == sp.SPLICE_ESHAPE
    assert entry(new=ints(5, 1, 0)) == sp.SPLICE_ESHAPE                   # more than T
    assert entry(new=ints(-1, 1, 0)) == sp.SPLICE_ESHAPE
    assert entry(new=None, steps=ints(97, 0, -1)) == sp.SPLICE_ESHAPE
    # nothing to do: finished cells (whatever their number of tokens says), or no tokens
    assert entry(steps=ints(-1, -7, -1), new=ints(99, -3, 0)) == sp.SPLICE_OK
    assert entry(new=ints(0, 0, 4)) == sp.SPLICE_OK


def test_attention_refusals():
    for name in ("q", "out"):
        assert attn(**{name: None}) == sp.SPLICE_EINVAL
        assert attn(**{name: FAKE + 8}) == sp.SPLICE_EINVAL
    for name in ("clean", "donor", "lse"):
        assert attn(**{name: None}) == sp.SPLICE_EINVAL
        assert attn(**{name: FAKE + 2}) == sp.SPLICE_EINVAL
    assert attn(LW=None) == sp.SPLICE_EINVAL
    assert attn(LW=ints(0, -1, 1, 2, 9, 0)) == sp.SPLICE_ESHAPE
    assert attn(sh=shape(donor_zero=True)) == sp.SPLICE_EINVAL            # a table with the ZERO donor
    assert attn(call=sp.make_call(4, 0, 0, 0.125)) == sp.SPLICE_ESHAPE
    assert attn(call=sp.make_call(1, 0, -1, 0.125)) == sp.SPLICE_ESHAPE
    for scale in (0.0, -1.0, float("inf"), float("nan"), 3e38):
        assert attn(call=sp.make_call(1, 0, 0, scale)) == sp.SPLICE_EINVAL
    assert attn(call=sp.make_call(1, 0, 0, 0.125, 100)) == sp.SPLICE_EINVAL
    long = shape(prompt_len=4096, span=(0, 0), n_cells=1)
    need = sp.splice_page_attn_workspace_bytes(long, sp.make_call(1, 0, 0, 0.125), sp.make_pages(99, 2, 1))
    assert need > 0
    one = dict(sh=long, pages=sp.make_pages(99, 2, 1), steps=ints(5), new=ints(1))
    assert attn(**one, ws=None) == sp.SPLICE_EWORKSPACE
    assert attn(**one, ws=FAKE + 128) == sp.SPLICE_EWORKSPACE
    assert attn(**one, bytes=512) == sp.SPLICE_EWORKSPACE
    with pytest.raises(sp.SpliceError):
        sp.splice_page_attn_workspace_bytes(shape(dtype="f32"), sp.make_call(1, 0, 0, 0.125), sp.make_pages(9, 2, 4))


def test_more_rows_than_a_launch_takes():
    sh = shape(n_cells=1, n_q_heads=65528, n_kv_heads=8191, head_dim=256, prompt_len=1 << 27, gen_capacity=1 << 20, span=(0, 0))
    pages = sp.make_pages(9, 1 << 14, 32768)
    assert attn(sh=sh, pages=pages, steps=ints(5), new=ints(32768), bytes=1 << 62) == sp.SPLICE_EUNSUPPORTED
    sh = shape(n_cells=256, n_q_heads=65528, n_kv_heads=8191, gen_capacity=1 << 20)
    many = (ctypes.c_int32 * 256)(*([5] * 256))
    assert attn(sh=sh, pages=pages, steps=many, new=None, LW=(ctypes.c_int32 * 512)(), bytes=1 << 62) == sp.SPLICE_EUNSUPPORTED


def test_append_refusals():
    for name in ("q", "k", "v", "q_out"):
        assert append(**{name: None}) == sp.SPLICE_EINVAL
        assert append(**{name: FAKE + 8}) == sp.SPLICE_EINVAL
    assert append(freq=None) == sp.SPLICE_EINVAL
    assert append(pos=FAKE + 4) == sp.SPLICE_EINVAL
    assert append(rope=sp.make_rope("half", 24)) == sp.SPLICE_ESHAPE
    assert append(rope=sp.make_rope("half", 128)) == sp.SPLICE_ESHAPE
    assert append(rope=sp.make_rope("half", 64, float("inf"))) == sp.SPLICE_EINVAL
    assert append(qs=504) == sp.SPLICE_ESHAPE
    assert append(ks=132) == sp.SPLICE_ESHAPE
    assert append(vs=(1 << 32) + 8) == sp.SPLICE_ESHAPE
    assert append(q_out=FAKE, qs=520) == sp.SPLICE_EINVAL                 # in place needs dense rows


def test_read_and_compact_refusals():
    assert read(rk=None) == sp.SPLICE_EINVAL
    assert read(rv=FAKE + 8) == sp.SPLICE_EINVAL
    assert compact(keep=None) == sp.SPLICE_EINVAL
    assert compact(steps=None) == sp.SPLICE_EINVAL
    assert compact(steps=ints(101, 0, 0)) == sp.SPLICE_ESHAPE
    assert compact(stride=9 * 2 * 68 * 64 - 16) == sp.SPLICE_EINVAL
    assert compact(stride=9 * 2 * 68 * 64 + 8) == sp.SPLICE_EINVAL
    assert compact(steps=ints(-1, -1, -2)) == sp.SPLICE_OK


def test_fork_refusals():
    for name in ("refs", "new_tables", "new_refs", "missing", "copied"):
        assert fork(**{name: None}) == sp.SPLICE_EINVAL
        assert fork(**{name: FAKE + 2}) == sp.SPLICE_EINVAL
    assert fork(parent=None) == sp.SPLICE_EINVAL
    assert fork(rows=None) == sp.SPLICE_EINVAL
    assert fork(want=None) == sp.SPLICE_EINVAL
    assert fork(new_tables=FAKE) == sp.SPLICE_EINVAL                      # in place
    assert fork(new_refs=FAKE) == sp.SPLICE_EINVAL
    assert fork(parent=ints(0, 3, -1)) == sp.SPLICE_ESHAPE
    assert fork(rows=ints(5, -1, 0)) == sp.SPLICE_ESHAPE
    assert fork(rows=ints(5, 5, 1), want=ints(9, 9, 9)) == sp.SPLICE_ESHAPE   # rows of nobody
    assert fork(want=ints(4, 9, 0)) == sp.SPLICE_ESHAPE                   # fewer than it takes over
    assert fork(want=ints(9, 129, 0)) == sp.SPLICE_ESHAPE                 # more than its table names
    assert fork(stride=16) == sp.SPLICE_EINVAL


def test_page_bytes():
    assert sp.splice_page_bytes(shape()) == 2 * 68 * 64
    with pytest.raises(sp.SpliceError):
        sp.splice_page_bytes(shape(head_dim=65))


@pytest.mark.parametrize("D", [64, 128, 256])
def test_every_byte_of_a_page_has_one_use(D):
    at = ref.places(np.arange(64)[:, None], np.arange(D), D)
    k, v, ks, vs = (np.broadcast_to(x, (64, D)) for x in at)
    used = np.concatenate([x.ravel() for x in (k[:, 0::2], v[:, 0::2], ks[:, 0::32], vs[:, 0::32])])
    assert sorted(used) == list(range(68 * D))
    for x in (k, v):
        assert (x[:, 0::2] == x[:, 1::2]).all()
    for x in (ks, vs):
        assert (x.reshape(64, -1, 32) == x[:, 0::32, None]).all()


def test_reference_quantisation():
    x = np.zeros((1, 32))
    x[0, :9] = 6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5.01
    codes, e = ref.quantised(x)
    assert e[0, 0] == 0 and list(ref.dequantised(codes, e)[0, :9]) == [6, 0, 1, 1, 2, 2, 4, 4, -6]
    codes, e = ref.quantised(x * 1.01)
    assert e[0, 0] == 1
    rng = np.random.default_rng(0)
    y = rng.standard_normal((5, 64)) * 2.0 ** rng.integers(-40, 40, (5, 1))
    codes, e = ref.quantised(y)
    assert (np.abs(ref.dequantised(codes, e) - y) <= np.repeat(2.0 ** e, 32, -1)).all()      # half of the widest step
    z = ref.dequantised(codes, e)
    again = ref.dequantised(*ref.quantised(z))
    assert (again == z).all()
    k, v = ref.rows_of(ref.page_of(rng.standard_normal((64, 128)), rng.standard_normal((64, 128))), 128)
    k2, v2 = ref.rows_of(ref.page_of(k, v), 128)
    assert (k == k2).all() and (v == v2).all()


def test_rows_alone():
    """Without q and q_out nothing is rotated; one of them alone is an error."""
    assert append(q=None) == append(q_out=None) == sp.SPLICE_EINVAL
    assert append(q=None, q_out=None, qs=0, k=None) == sp.SPLICE_EINVAL
    assert append(q=None, q_out=None, qs=0, new=ints(0, 0, 0)) == sp.SPLICE_OK
