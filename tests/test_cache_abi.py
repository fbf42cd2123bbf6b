"""Host-side checks of the paged cache's C ABI: struct layouts, plans, every
refusal of the calls (fake device pointers, refused before a launch), and the
tiles that a launch's workgroups cover."""
import ctypes
import os
import random
import subprocess

import pytest
import torch

import cache_reference as R
import paper_2310_11960_amd as F
from paper_2310_11960_amd import build as hip_build

V = F.fma_view_t
MB = 1 << 20


def _desc(**kw):
    d = dict(dtype=F.FMA_BF16, heads=4, kv_heads=2, head_dim=64, block=64, max_seq_len=4096, rank=1, weights_per_head=1,
             norm=0, softmax_scale=0.0)
    d.update(kw)
    x = F.fma_cache_desc_t(**d)
    x.struct_size = ctypes.sizeof(F.fma_cache_desc_t)
    return x


def _status(fn, *args):
    with pytest.raises(F.FmaError) as e:
        fn(*args)
    return e.value.status


@pytest.mark.parametrize("name", ["fma_cache_desc_t", "fma_cache_batch_t"])
def test_struct_layouts_match_the_header(name, tmp_path):
    t = getattr(F, name)
    names = [f[0] for f in t._fields_]
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "fma.h"\nint main(void){\n'
    src += 'printf("size %%zu\\n", sizeof(%s));\n' % name
    for n in names:
        src += 'printf("%s %%zu\\n", offsetof(%s, %s));\n' % (n, name, n)
    c, exe = str(tmp_path / "probe.c"), str(tmp_path / "probe")
    open(c, "w").write(src + "return 0;}\n")
    subprocess.run(["gcc", "-I", os.path.dirname(F.HEADER_PATH), c, "-o", exe], check=True)
    out = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()
    got = dict(zip(out[0::2], map(int, out[1::2])))
    assert got["size"] == ctypes.sizeof(t)
    for n in names:
        assert got[n] == getattr(t, n).offset, n


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), F.FMA_ERR_ARG), (dict(heads=0), F.FMA_ERR_SHAPE), (dict(kv_heads=3), F.FMA_ERR_SHAPE),
    (dict(heads=1 << 15), F.FMA_ERR_SHAPE), (dict(head_dim=96), F.FMA_ERR_UNSUPPORTED), (dict(block=0), F.FMA_ERR_SHAPE),
    (dict(block=48), F.FMA_ERR_UNSUPPORTED), (dict(block=512), F.FMA_ERR_UNSUPPORTED),
    (dict(max_seq_len=0), F.FMA_ERR_SHAPE), (dict(max_seq_len=1 << 31), F.FMA_ERR_SHAPE),
    (dict(block=16, max_seq_len=1 << 30), F.FMA_ERR_UNSUPPORTED), (dict(rank=-1), F.FMA_ERR_ARG),
    (dict(rank=17), F.FMA_ERR_UNSUPPORTED), (dict(weights_per_head=2), F.FMA_ERR_ARG), (dict(norm=5), F.FMA_ERR_ARG),
    (dict(norm=F.FMA_NORM_PER_LEVEL), F.FMA_ERR_UNSUPPORTED), (dict(softmax_scale=float("inf")), F.FMA_ERR_ARG)])
def test_plan_refusals(change, status):
    assert _status(F.fma_cache_plan, _desc(**change)) == status


@pytest.mark.parametrize("r", [16, 64, 192, 256])
@pytest.mark.parametrize("blocks", [1, 2, 3, 4, 5, 64, 65, 512])
def test_sizes_are_those_of_the_dense_plan(r, blocks):
    for max_len in (r * blocks, r * blocks - r + 1):
        c = F.FMACache(2, max_len, block=r, rank=2)
        p = F.FMA(ndim=1, heads=2, seq_len=r * blocks, block=r, rank=2, causal=True)
        assert c.blocks == blocks and c.weights_len == p.weights_len == R.weight_len(max_len, r, 2)
        assert c.sets == 2 * max(p.levels - 1, 0)
    assert F.fma_cache_sizes(c.handle) == (c.sets, c.weights_len, c.blocks)


def test_plan_struct_size_and_nulls():
    d = _desc()
    d.struct_size += 8
    assert _status(F.fma_cache_plan, d) == F.FMA_ERR_ARG
    assert F.library().fma_cache_plan(None, None) == F.FMA_ERR_NULL
    assert F.library().fma_cache_sizes(None, None, None, None) == F.FMA_ERR_NULL
    F.fma_cache_destroy(None)
    F.fma_cache_destroy(F.fma_cache_plan(_desc(rank=0)))


def _batch(**kw):
    b = dict(k_pages=MB * 16, v_pages=MB * 32, summaries=MB * 48, num_pages=20, num_summaries=20, page_table=MB * 64,
             summary_table=MB * 65, table_stride=64, cu_tokens=MB * 66, start=MB * 67, sequences=3, max_chunk=30, rows=50)
    b.update(kw)
    return F.fma_cache_batch_t(**b)


def _views():
    return {"q": V(MB * 80, 0, 64, 256), "k": V(MB * 81, 0, 64, 128), "v": V(MB * 82, 0, 64, 128),
            "out": V(MB * 83, 0, 64, 256)}


@pytest.fixture
def plan():
    p = F.fma_cache_plan(_desc())
    yield p
    F.fma_cache_destroy(p)


def _calls(plan, batch, views, wk=MB * 90, wv=MB * 91):
    """Status of append, attend and step."""
    x = views
    return [_status(F.fma_cache_append, plan, batch, x["k"], x["v"], wk, wv, 0),
            _status(F.fma_cache_attend, plan, batch, x["q"], x["out"], 0),
            _status(F.fma_cache_step, plan, batch, x["q"], x["k"], x["v"], wk, wv, x["out"], 0)]


@pytest.mark.parametrize("change,status", [
    (dict(sequences=-1), F.FMA_ERR_SHAPE), (dict(max_chunk=-1), F.FMA_ERR_SHAPE), (dict(rows=-1), F.FMA_ERR_SHAPE),
    (dict(num_pages=-1), F.FMA_ERR_SHAPE), (dict(num_summaries=-1), F.FMA_ERR_SHAPE), (dict(table_stride=-1), F.FMA_ERR_SHAPE),
    (dict(rows=(1 << 21) + 1), F.FMA_ERR_SHAPE), (dict(sequences=(1 << 20) + 1), F.FMA_ERR_SHAPE),
    (dict(num_pages=1 << 31), F.FMA_ERR_SHAPE), (dict(k_pages=None), F.FMA_ERR_NULL), (dict(v_pages=None), F.FMA_ERR_NULL),
    (dict(summaries=None), F.FMA_ERR_NULL), (dict(page_table=None), F.FMA_ERR_NULL), (dict(summary_table=None), F.FMA_ERR_NULL),
    (dict(cu_tokens=None), F.FMA_ERR_NULL), (dict(start=None), F.FMA_ERR_NULL), (dict(k_pages=MB * 16 + 8), F.FMA_ERR_ALIGN),
    (dict(summaries=MB * 48 + 4), F.FMA_ERR_ALIGN), (dict(start=MB + 2), F.FMA_ERR_ALIGN),
    (dict(v_pages=MB * 16 + 16384), F.FMA_ERR_ARG), (dict(summaries=MB * 16), F.FMA_ERR_ARG)])
def test_batch_refusals(plan, change, status):
    assert _calls(plan, _batch(**change), _views()) == [status] * 3


def test_call_refusals(plan):
    b, x = _batch(), _views()
    assert _calls(None, b, x) == [F.FMA_ERR_NULL] * 3
    assert F.library().fma_cache_append(plan, None, F._ref(x["k"]), F._ref(x["v"]), None, None, None) == F.FMA_ERR_NULL
    step = lambda **kw: _status(F.fma_cache_step, plan, b, *[kw.get(n, x.get(n)) for n in ("q", "k", "v")],  # noqa: E731
                                kw.get("wk", MB * 90), kw.get("wv", MB * 91), kw.get("out", x["out"]), 0)
    for n in ("q", "k", "v", "out"):
        assert step(**{n: None}) == F.FMA_ERR_NULL
        assert step(**{n: V(0, 0, 64, 256)}) == F.FMA_ERR_NULL
        assert step(**{n: V(x[n].data + 4, 0, 64, 256)}) == F.FMA_ERR_ALIGN
        assert step(**{n: V(x[n].data, 0, 64, 260)}) == F.FMA_ERR_ALIGN
        assert step(**{n: V(x[n].data, 0, 64, -256)}) == F.FMA_ERR_SHAPE
        assert step(**{n: V(MB * 16 + 64, 0, 64, 256)}) == F.FMA_ERR_ARG        # inside a pool
    assert step(wk=None) == F.FMA_ERR_NULL and step(wv=MB + 2) == F.FMA_ERR_ALIGN
    assert step(out=V(MB * 83, 0, 64, 128)) == F.FMA_ERR_ARG                    # output rows share elements
    assert step(out=V(x["q"].data + 128, 0, 64, 256)) == F.FMA_ERR_ARG
    assert step(out=V(x["k"].data, 0, 64, 256)) == F.FMA_ERR_ARG
    assert _status(F.fma_cache_append, plan, b, None, x["v"], MB, MB, 0) == F.FMA_ERR_NULL
    assert _status(F.fma_cache_append, plan, b, x["k"], None, MB, MB, 0) == F.FMA_ERR_NULL
    assert _status(F.fma_cache_attend, plan, b, None, x["out"], 0) == F.FMA_ERR_NULL
    assert _status(F.fma_cache_attend, plan, b, x["q"], None, 0) == F.FMA_ERR_NULL


@pytest.mark.parametrize("change", [dict(sequences=0), dict(rows=0), dict(max_chunk=0)])
def test_calls_without_tokens_need_nothing(plan, change):
    b = F.fma_cache_batch_t(sequences=2, rows=2, max_chunk=2)
    for n, v in change.items():
        setattr(b, n, v)
    x = _views()
    F.fma_cache_append(plan, b, x["k"], x["v"], None, None, 0)
    F.fma_cache_attend(plan, b, x["q"], x["out"], 0)
    F.fma_cache_step(plan, b, x["q"], x["k"], x["v"], None, None, x["out"], 0)


def test_object_refusals():
    op = F.FMACache(4, 4096, kv_heads=2)
    cpu = -1      # (the device number of CPU tensors)
    pages = op.new_pages(3, 3, "cpu")
    z = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    b = F.CacheBatch(z(3), z(2), z(2, 5), z(2, 5), 4)
    k = torch.zeros(7, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(F.FmaError, match="GPU"):
        op.append(k, k, None, None, pages, b)
    raw = op._batch(pages, b, 7, cpu)
    assert (raw.num_pages, raw.num_summaries, raw.table_stride, raw.sequences, raw.max_chunk, raw.rows) == (3, 3, 5, 2, 4, 7)
    for bad, status in ((b._replace(start=z(3)), F.FMA_ERR_SHAPE), (b._replace(cu_tokens=z(2)), F.FMA_ERR_SHAPE),
                        (b._replace(page_table=z(2, 5).long()), F.FMA_ERR_ARG), (b._replace(page_table=z(3, 5)), F.FMA_ERR_SHAPE),
                        (b._replace(summary_table=z(2, 4)), F.FMA_ERR_SHAPE), (b._replace(summary_table=None), F.FMA_ERR_NULL),
                        (b._replace(page_table=z(5, 2).t()), F.FMA_ERR_SHAPE), (b._replace(page_table=z(5)), F.FMA_ERR_SHAPE)):
        assert _status(op._batch, pages, bad, 7, cpu) == status
    for bad, status in ((pages._replace(k=pages.k.float()), F.FMA_ERR_ARG), (pages._replace(v=pages.v[:2]), F.FMA_ERR_SHAPE),
                        (pages._replace(summaries=None), F.FMA_ERR_NULL),
                        (pages._replace(summaries=pages.summaries[..., :32]), F.FMA_ERR_SHAPE)):
        assert _status(op._batch, bad, b, 7, cpu) == status
    assert _status(op._rows, k, "k", 4, 7, cpu) == F.FMA_ERR_SHAPE
    assert _status(op._rows, k.float(), "k", 2, 7, cpu) == F.FMA_ERR_ARG
    assert _status(op._rows, torch.zeros(7, 64, 2, dtype=torch.bfloat16).transpose(1, 2), "k", 2, 7, cpu) == F.FMA_ERR_SHAPE
    w = torch.zeros(2, op.weights_len)
    assert op._weights(w, w, cpu)[0] is w
    assert _status(op._weights, None, w, cpu) == F.FMA_ERR_NULL
    assert _status(op._weights, w[0], w, cpu) == F.FMA_ERR_SHAPE


@pytest.fixture(scope="module")
def tiling(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("host_cache") / "host_cache.so")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run([hip_build._hipcc(), "-O1", "-std=c++17", "--offload-arch=gfx950", "--cuda-host-only", "-fPIC", "-shared",
                    "-I", hip_build.INCLUDE, "-I", hip_build.CSRC, os.path.join(here, "host_cache.hip"), "-o", so], check=True)
    return ctypes.CDLL(so)


def test_launches_cover_every_tile(tiling):
    """However the sequences lie, their tiles number no more than the workgroups
    launched, nor any one sequence's than its share; tiles do not cross
    blocks and hold at most tm positions."""
    rng = random.Random(1)
    out = (ctypes.c_longlong * 4)()
    searched = direct = 0
    for _ in range(4000):
        r = rng.choice([16, 32, 64, 128, 192, 256])
        tm = rng.choice([1, 2, 10, 16, 32, 128, 256, r])
        S = rng.choice([1, 2, 5, 60])
        most = rng.choice([1, 2, 7, r, r + 1, 5 * r])
        lens = [rng.choice([0, 1, rng.randrange(most + 1), most]) for _ in range(S)]
        starts = [rng.randrange(20 * r) for _ in range(S)]
        rows = max(1, sum(lens) + rng.choice([0, 3]))
        tiling.host_cache_tiling(r, S, most, rows, tm, out)
        t, tpb, per, units = out[:]
        of = lambda p: tiling.host_cache_tile_of(r, t, tpb, p)  # noqa: E731
        counts = [of(s + n - 1) - of(s) + 1 if n else 0 for s, n in zip(starts, lens)]
        assert t == min(tm, r) and tpb == -(-r // t)
        if per:
            direct += 1
            assert units == per * S and max(counts) <= per
        else:
            searched += 1
            assert sum(counts) <= units
        assert units <= 2 * rows + 64
    assert searched > 100 and direct > 100
    for r, tm in ((192, 128), (256, 10), (16, 16)):
        tpb = -(-r // tm)
        tiles = [tiling.host_cache_tile_of(r, tm, tpb, p) for p in range(3 * r)]
        assert tiles == [p // r * tpb + p % r // tm for p in range(3 * r)]


def test_tiles_of_query_heads(tiling):
    """Every query head has one workgroup, which holds at most 32 of them; a
    tile holds at most 128 rows and a block few tiles more than it must."""
    out = (ctypes.c_int * 4)()
    for r in (16, 32, 64, 128, 192, 256):
        for group in range(1, 200):
            tiling.host_cache_route(r, group, 1, r, 10 * r, 64, 1, 256, out)
            _, gs, split, tm = out[:]
            assert 1 <= gs <= 32 and (split - 1) * gs < group <= split * gs
            assert 1 <= tm <= r and tm * gs <= 128
            assert -(-r // tm) <= 2 * -(-r * gs // 128)


BF32, BF64, BF128, F32, F64, F128 = (32, 1), (64, 1), (128, 1), (32, 0), (64, 0), (128, 0)


@pytest.mark.parametrize("args,kind,route", [
    ((128, 1, 16, 1, 1), BF64, 0), ((128, 2, 4, 1, 100), BF64, 0), ((128, 1, 8, 2, 40), BF32, 0),   # few rows per key head
    ((128, 4, 4, 1, 100), BF128, 0), ((128, 1, 8, 4, 40), F64, 0), ((128, 4, 4, 1, 100), BF64, 1),
    ((128, 5, 4, 1, 100), F128, 1), ((128, 1, 16, 5, 2000), BF64, 1), ((128, 8, 16, 4, 9000), BF128, 1),   # one tile of 32
    ((128, 1, 16, 128, 1024), BF64, 1), ((128, 1, 16, 4096, 1792), BF32, 1), ((128, 1, 16, 4096, 512), BF128, 1),   # all at once
    ((128, 1, 16, 4096, 1280), F64, 1), ((128, 1, 16, 4096, 1024), F128, 1), ((128, 1, 16, 4096, 1792), F32, 1),
    ((128, 1, 16, 128, 1152), BF64, 2), ((128, 1, 16, 4096, 2048), BF32, 2), ((128, 1, 16, 4096, 640), BF128, 2),
    ((128, 1, 16, 4096, 1536), F64, 2), ((128, 1, 16, 4096, 1152), F128, 2),
    ((64, 4, 4, 2500, 8000), BF64, 2), ((16, 1, 16, 400, 400), BF64, 2)])
def test_routes(tiling, args, kind, route):
    out = (ctypes.c_int * 4)()
    r, group, kv, chunk, rows = args
    tiling.host_cache_route(r, group, kv, chunk, rows, *kind, 256, out)
    assert out[0] == route
