"""Host-only checks of the key/value cache calls: sizes, and refusals before the GPU is touched."""
import ctypes

import pytest
import torch

from paper_2309_14717_b200 import binding as Q
from paper_2309_14717_b200 import build as _build

p, r = ctypes.c_void_p, ctypes.byref


@pytest.fixture(scope="module", autouse=True)
def _built():
    _build.build()


@pytest.fixture
def at():
    buf = ctypes.create_string_buffer(64)          # host memory: must never be dereferenced
    a16 = (ctypes.addressof(buf) + 15) // 16 * 16
    yield a16
    del buf


GOOD = (8, 2, 128, 64, 100)


def test_sizes():
    d = Q.kv_desc(*GOOD)
    assert Q.qalora_kv_cache_bytes(d) == (100 * 2 * 2 * 64 * 128, 100 * 2 * 2 * 4, 100 * 2 * 64 * 4)
    few = Q.qalora_kv_attention_workspace_bytes(d, 4, 4, 1, 1000, False)
    scored = Q.qalora_kv_attention_workspace_bytes(d, 4, 4, 1, 1000, True)
    assert 0 < few < scored
    assert Q.qalora_kv_attention_workspace_bytes(d, 0, 0, 0, 0, True) > 0


@pytest.mark.parametrize("desc,status", [
    ((0, 2, 128, 64, 100), -1), ((8, 0, 128, 64, 100), -1), ((8, 2, 0, 64, 100), -1), ((8, 2, 128, -64, 100), -1), ((8, 2, 128, 64, 0), -1),
    ((9, 2, 128, 64, 100), -3), ((2, 8, 128, 64, 100), -3), ((2048, 2, 128, 64, 100), -3), ((8, 2, 96, 64, 100), -3),
    ((8, 2, 256, 64, 100), -3), ((8, 2, 128, 48, 100), -3), ((8, 2, 128, 256, 100), -3), ((8, 8, 128, 128, 1 << 20), -3),
])
def test_bad_descriptors(desc, status):
    with pytest.raises(Q.QaloraError) as e:
        Q.qalora_kv_cache_bytes(Q.kv_desc(*desc))
    assert e.value.status == status
    assert Q.load().qalora_kv_cache_bytes(None, None, None, None) == -2


def _append(at, **change):
    v = dict(d=Q.kv_desc(*GOOD), batch=3, m=6, max_new=2, starts=at, lens=at, table=at, width=4, k=at, ks=256, v=at, vs=256, codes=at,
             scales=at, score=None, flag=None)
    v.update(change)
    return Q.load().qalora_kv_append(r(v["d"]), v["batch"], v["m"], v["max_new"], p(v["starts"]), p(v["lens"]), p(v["table"]), v["width"],
                                     p(v["k"]), v["ks"], p(v["v"]), v["vs"], p(v["codes"]), p(v["scales"]), p(v["score"]), p(v["flag"]), None)


@pytest.mark.parametrize("change,status", [
    (dict(batch=-1), -1), (dict(batch=65536), -1), (dict(m=-1), -1), (dict(m=(1 << 22) + 1), -1), (dict(max_new=-1), -1), (dict(max_new=7), -1),
    (dict(width=-1), -1), (dict(ks=248), -1), (dict(ks=260), -1), (dict(vs=0), -1), (dict(vs=1 << 50), -1),
    (dict(starts=None), -2), (dict(lens=None), -2), (dict(table=None), -2), (dict(k=None), -2), (dict(v=None), -2), (dict(codes=None), -2),
    (dict(scales=None), -2), (dict(batch=0, starts=None), 0), (dict(m=0, max_new=0, k=None), 0), (dict(max_new=0), 0), (dict(width=0), 0),
])
def test_append_refusals(at, change, status):
    assert _append(at, **change) == status


@pytest.mark.parametrize("name,off", [("starts", 2), ("lens", 1), ("table", 2), ("k", 8), ("v", 2), ("codes", 4), ("scales", 4), ("score", 4), ("flag", 2)])
def test_append_alignment(at, name, off):
    assert _append(at, **{name: at + off}) == -4


def _attention(at, **change):
    v = dict(d=Q.kv_desc(*GOOD), batch=3, m=6, max_new=2, max_len=200, starts=at, lens=at, table=at, width=4, q=at, qs=1024, codes=at,
             scales=at, scale=0.1, out=at, lse=None, sin=None, sout=None, ws=at, bytes=1 << 40)
    v.update(change)
    return Q.load().qalora_kv_attention(r(v["d"]), v["batch"], v["m"], v["max_new"], v["max_len"], p(v["starts"]), p(v["lens"]), p(v["table"]),
                                        v["width"], p(v["q"]), v["qs"], p(v["codes"]), p(v["scales"]), v["scale"], p(v["out"]), p(v["lse"]),
                                        p(v["sin"]), p(v["sout"]), p(v["ws"]), v["bytes"], None)


@pytest.mark.parametrize("change,status", [
    (dict(batch=-1), -1), (dict(m=-1), -1), (dict(max_new=7), -1), (dict(max_len=-1), -1), (dict(width=-1), -1), (dict(qs=1016), -1),
    (dict(qs=1028), -1), (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1),
    (dict(starts=None), -2), (dict(lens=None), -2), (dict(table=None), -2), (dict(q=None), -2), (dict(codes=None), -2), (dict(scales=None), -2),
    (dict(out=None), -2), (dict(ws=None), -2), (dict(sin=16), -2), (dict(bytes=64), -5), (dict(batch=0, q=None), 0), (dict(m=0, max_new=0), 0),
])
def test_attention_refusals(at, change, status):
    if change.get("sin"):
        change = dict(sin=at)
    assert _attention(at, **change) == status


@pytest.mark.parametrize("name,off", [("starts", 2), ("lens", 2), ("table", 1), ("q", 8), ("codes", 8), ("scales", 4), ("out", 4), ("lse", 4),
                                      ("sout", 4), ("ws", 4)])
def test_attention_alignment(at, name, off):
    assert _attention(at, **{name: at + off}) == -4


def test_attention_workspace_is_checked_for_the_size_with_scores(at):
    d = Q.kv_desc(*GOOD)
    plain = Q.qalora_kv_attention_workspace_bytes(d, 3, 6, 2, 200, False)
    assert _attention(at, bytes=plain, sout=at) == -5


def _evict(at, **change):
    v = dict(d=Q.kv_desc(*GOOD), batch=3, max_len=200, budget=100, recent=10, lens=at, table=at, width=4, codes=at, scales=at, score=at, dst=at,
             dst_width=2, dst_lens=at, kept=at)
    v.update(change)
    return Q.load().qalora_kv_evict(r(v["d"]), v["batch"], v["max_len"], v["budget"], v["recent"], p(v["lens"]), p(v["table"]), v["width"],
                                    p(v["codes"]), p(v["scales"]), p(v["score"]), p(v["dst"]), v["dst_width"], p(v["dst_lens"]), p(v["kept"]), None)


@pytest.mark.parametrize("change,status", [
    (dict(batch=-1), -1), (dict(max_len=-1), -1), (dict(budget=0), -1), (dict(recent=-1), -1), (dict(recent=101), -1), (dict(width=-1), -1),
    (dict(dst_width=1), -1), (dict(lens=None), -2), (dict(table=None), -2), (dict(codes=None), -2), (dict(scales=None), -2),
    (dict(score=None), -2), (dict(dst=None), -2), (dict(dst_lens=None), -2), (dict(kept=None), -2), (dict(batch=0, lens=None), 0),
])
def test_evict_refusals(at, change, status):
    assert _evict(at, **change) == status


@pytest.mark.parametrize("name,off", [("lens", 2), ("table", 2), ("codes", 8), ("scales", 4), ("score", 4), ("dst", 2), ("dst_lens", 1), ("kept", 2)])
def test_evict_alignment(at, name, off):
    assert _evict(at, **{name: at + off}) == -4


def test_read_refusals(at):
    def read(batch=3, m=6, max_new=2, starts=at, first=at, table=at, width=4, codes=at, scales=at, k=at, v=at):
        return Q.load().qalora_kv_read(r(Q.kv_desc(*GOOD)), batch, m, max_new, p(starts), p(first), p(table), width, p(codes), p(scales), p(k),
                                       p(v), 0, None)
    assert read(batch=-1) == -1 and read(m=-2) == -1 and read(max_new=7) == -1 and read(width=-1) == -1
    assert read(starts=None) == -2 and read(first=None) == -2 and read(table=None) == -2 and read(codes=None) == -2 and read(scales=None) == -2
    assert read(k=at + 8) == -4 and read(v=at + 4) == -4 and read(codes=at + 2) == -4 and read(first=at + 1) == -4
    assert read(k=None, v=None) == 0 and read(batch=0) == 0 and read(m=0, max_new=0) == 0


def test_binding_refuses_wrong_tensors():
    d = Q.kv_desc(*GOOD)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    codes, scales = torch.zeros((100, 2, 2, 64, 128), dtype=torch.int8), torch.zeros((100, 2, 2))
    k = torch.zeros((6, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="lens"):
        Q.qalora_kv_append(d, 2, i32(4), torch.zeros(3), i32(3, 4), k, k, codes, scales)
    with pytest.raises(ValueError, match="starts"):
        Q.qalora_kv_append(d, 2, i32(3), i32(3), i32(3, 4), k, k, codes, scales)
    with pytest.raises(ValueError, match="table"):
        Q.qalora_kv_append(d, 2, i32(4), i32(3), i32(2, 4), k, k, codes, scales)
    with pytest.raises(ValueError, match="codes"):
        Q.qalora_kv_append(d, 2, i32(4), i32(3), i32(3, 4), k, k, codes[:50], scales)
    with pytest.raises(ValueError, match="k "):
        Q.qalora_kv_append(d, 2, i32(4), i32(3), i32(3, 4), k.float(), k, codes, scales)
    with pytest.raises(ValueError, match="CUDA"):
        Q.qalora_kv_append(d, 2, i32(4), i32(3), i32(3, 4), k, k, codes, scales)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        Q.qalora_kv_read(d, 2, i32(4), i32(3), i32(3, 4), codes, scales, k.half(), None)
