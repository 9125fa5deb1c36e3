"""Refusals of the paged key-value cache's calls: what they check on the host, before any device is touched.
Addresses are made up; nothing is read through them."""
import ctypes as C
import math
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20                       # an aligned address


@pytest.fixture(scope="module")
def td():
    from paper_2507_19017_b200 import build, binding
    build.build()
    return binding


def cache(td, **kw):
    v = dict(dtype=td.BF16, n_pages=20, page_size=16, n_layers=2, n_heads=4, dim=64, layer_stride=20 * 16 * 256, page_stride=16 * 256,
             token_stride=256, head_stride=64, keys=A, values=2 * A, max_seqs=6, max_pages=5, table=A, length=A, holders=A, status=A,
             workspace=A, workspace_bytes=1 << 30, device=0, reserved=0)
    v.update(kw)
    return td.TdCache(**v)


def extend(td, add=A, cu=A, **kw):
    return td.lib().td_cache_extend(C.addressof(c := cache(td, **kw)), add, cu, None)


def fork(td, parent=A, **kw):
    return td.lib().td_cache_fork(C.addressof(c := cache(td, **kw)), parent, None)


def free(td, release=A, **kw):
    return td.lib().td_cache_free(C.addressof(c := cache(td, **kw)), release, None)


def compact(td, used=A, moved=A, **kw):
    return td.lib().td_cache_compact(C.addressof(c := cache(td, **kw)), used, moved, None)


OWN = dict(layer=1, n_rows=3, n_heads=8, group=1, window=0, scale=0.125, seqs=A, q=A, q_row_stride=512, q_head_stride=64, out=A,
           out_row_stride=512, out_head_stride=64, lse=A, workspace=A, workspace_bytes=1 << 30)
ROWS = dict(layer=1, n_rows=3, keys=A, values=A, row_stride=256, head_stride=64, cu=A)


def attend(td, **kw):
    """Names that both structs have (n_heads, workspace) are the attention's; the cache's are given as cache_<name>."""
    v = dict(OWN, **{k: x for k, x in kw.items() if k in OWN})
    c = cache(td, **{k.removeprefix("cache_"): x for k, x in kw.items() if k not in OWN})
    return td.lib().td_cache_attention(td.TdCacheAttentionArgs(cache=C.pointer(c), reserved=0, reserved2=0, **v), None)


def write(td, **kw):
    v = dict(ROWS, **{k: x for k, x in kw.items() if k in ROWS})
    c = cache(td, **{k.removeprefix("cache_"): x for k, x in kw.items() if k not in ROWS})
    return td.lib().td_cache_write(td.TdCacheWriteArgs(cache=C.pointer(c), **v), None)


TABLES = [dict(dtype=0), dict(dtype=9), dict(page_size=0), dict(page_size=1 << 16), dict(n_pages=1 << 31), dict(max_seqs=1 << 24),
          dict(max_pages=1 << 28), dict(table=None), dict(length=None), dict(holders=None), dict(table=A + 2), dict(length=A + 1),
          dict(holders=A + 2), dict(status=A + 1), dict(n_pages=1 << 30, page_size=1 << 10)]
POOL = [dict(n_layers=0), dict(n_layers=1 << 16), dict(cache_n_heads=0), dict(cache_n_heads=1 << 16), dict(dim=0), dict(dim=1 << 16),
        dict(layer_stride=-1), dict(page_stride=-16), dict(token_stride=-16), dict(cache_head_stride=-16), dict(cache_keys=A + 1),
        dict(cache_values=A + 1), dict(cache_keys=None), dict(cache_values=None), dict(page_size=1 << 15, cache_n_heads=1 << 12, dim=256),
        dict(cache_keys=None, cache_values=None)]


def plain(bad):
    return {k.removeprefix("cache_"): v for k, v in bad.items()}


@pytest.mark.parametrize("bad", TABLES + [dict(add=A + 2), dict(cu=A + 1)] + POOL[:-1], ids=str)
def test_extend_refuses(td, bad):
    assert extend(td, **plain(bad)) == td.EINVAL


@pytest.mark.parametrize("bad", TABLES + POOL[:-1], ids=str)
def test_free_refuses(td, bad):
    assert free(td, **plain(bad)) == td.EINVAL


@pytest.mark.parametrize("bad", TABLES + POOL + [dict(parent=None), dict(parent=A + 2)], ids=str)
def test_fork_refuses(td, bad):
    assert fork(td, **plain(bad)) == td.EINVAL


@pytest.mark.parametrize("bad", TABLES + POOL + [dict(used=A + 2), dict(moved=A + 1)], ids=str)
def test_compact_refuses(td, bad):
    assert compact(td, **plain(bad)) == td.EINVAL


@pytest.mark.parametrize("bad", TABLES + POOL + [dict(layer=2), dict(n_rows=1 << 31), dict(keys=None), dict(values=None), dict(cu=None), dict(keys=A + 1),
                                                 dict(values=A + 1), dict(cu=A + 2), dict(row_stride=-1), dict(head_stride=-64)], ids=str)
def test_write_refuses(td, bad):
    assert write(td, **bad) == td.EINVAL


@pytest.mark.parametrize("bad", TABLES + POOL + [
    dict(layer=2), dict(n_rows=1 << 24), dict(n_heads=0), dict(n_heads=6), dict(n_heads=1 << 16), dict(group=0), dict(scale=math.nan),
    dict(scale=math.inf), dict(q=None), dict(out=None), dict(q=A + 8), dict(out=A + 8), dict(lse=A + 2), dict(seqs=A + 2), dict(q_row_stride=-512),
    dict(q_row_stride=516), dict(q_head_stride=-64), dict(q_head_stride=68), dict(out_row_stride=516), dict(out_head_stride=60), dict(out_head_stride=68), dict(out_head_stride=0),
    dict(out_row_stride=504), dict(dim=264), dict(dim=60), dict(page_stride=16 * 256 + 4), dict(token_stride=260), dict(cache_head_stride=68),
    dict(layer_stride=20 * 16 * 256 + 4), dict(cache_keys=A + 8), dict(cache_values=A + 8)], ids=str)
def test_attention_refuses(td, bad):
    assert attend(td, **bad) == td.EINVAL


def test_workspaces_are_checked(td):
    need = td.lib().td_cache_workspace_bytes(20, 6)
    for call in (extend, fork, compact):
        for bad in (dict(workspace=None), dict(workspace=A + 128), dict(workspace_bytes=need - 1)):
            assert call(td, **bad) == td.EWORKSPACE
    need = td.lib().td_cache_attention_workspace_bytes(3, 8, 64)
    for bad in (dict(workspace=None), dict(workspace=A + 128), dict(workspace_bytes=need - 1)):
        assert attend(td, **bad) == td.EWORKSPACE
    for call in (td.lib().td_cache_workspace_bytes, lambda a, b: td.lib().td_cache_attention_workspace_bytes(a, b, 128)):
        sizes = [call(a, b) for a in (0, 1, 7, 2000, 2049, 70000, 10 ** 6) for b in (0, 1, 16, 1025, 30000)]
        assert all(sizes)
        for i in range(7):
            assert sizes[5 * i:5 * i + 5] == sorted(sizes[5 * i:5 * i + 5])
        for i in range(5):
            assert sizes[i::5] == sorted(sizes[i::5])
    assert td.lib().td_cache_workspace_bytes(1 << 31, 1) == td.lib().td_cache_workspace_bytes(1, 1 << 24) == 0
    assert td.lib().td_cache_attention_workspace_bytes(1 << 24, 1, 64) == td.lib().td_cache_attention_workspace_bytes(1, 1, 257) == 0
    assert td.lib().td_cache_attention_workspace_bytes(1, 1 << 16, 64) == 0


def test_null_arguments_and_empty_calls(td):
    L = td.lib()
    assert L.td_cache_extend(None, None, None, None) == L.td_cache_fork(None, None, None) == td.EINVAL
    assert L.td_cache_free(None, None, None) == L.td_cache_compact(None, None, None, None) == td.EINVAL
    assert L.td_cache_write(None, None) == L.td_cache_attention(None, None) == td.EINVAL
    none = dict(max_seqs=0, table=None, length=None)
    assert extend(td, cu=None, **none) == fork(td, parent=None, **none) == free(td, **none) == td.OK
    assert compact(td, used=None, n_pages=0, holders=None, keys=None, values=None) == td.OK
    assert write(td, n_rows=0, keys=None, values=None, cu=None) == attend(td, n_rows=0, q=None, out=None) == td.OK


def test_a_call_without_a_device_says_so(td):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for call in (extend, fork, free, compact, write, attend):
        assert call(td) == td.ECUDA
    assert extend(td, keys=None, values=None) == free(td, keys=None, values=None) == td.ECUDA         # tables alone will do
    assert fork(td, parent=A, page_size=7, dim=3, n_heads=3) == td.ECUDA


def test_struct_layouts_match_the_header(td, tmp_path):
    names = {"td_cache": td.TdCache, "td_cache_write_args": td.TdCacheWriteArgs, "td_cache_attention_args": td.TdCacheAttentionArgs}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "td.h"', "int main(void) {"]
    for n, s in names.items():
        lines.append(f'printf("%zu\\n", sizeof({n}));')
        lines += [f'printf("%zu\\n", offsetof({n}, {f[0]}));' for f in s._fields_]
    (tmp_path / "o.c").write_text("\n".join(lines + ["return 0; }"]))
    exe = tmp_path / "o"
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(tmp_path / "o.c")])
    got = list(map(int, subprocess.check_output([str(exe)]).split()))
    want = [v for s in names.values() for v in [C.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]]
    assert got == want


class OnDevice:
    """What the binding asks of a tensor, for one that would be on a device."""

    def __init__(self, dtype, *shape, strides=None, device=0):
        self.dtype, self.shape, self.device, self.strides = dtype, shape, device, strides

    def get_device(self):
        return self.device

    def stride(self):
        if self.strides:
            return self.strides
        return tuple(math.prod(self.shape[i + 1:]) for i in range(len(self.shape)))

    def numel(self):
        return math.prod(self.shape)

    def is_contiguous(self):
        return self.strides is None

    def data_ptr(self):
        return A


def some_cache(td, monkeypatch, **kw):
    import torch
    for name in ("zeros", "empty"):
        real = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, device=None, real=real, **k: real(*a, **k))
    i32, bf16 = torch.int32, torch.bfloat16
    v = dict(keys=OnDevice(bf16, 2, 20, 16, 4, 64), values=OnDevice(bf16, 2, 20, 16, 4, 64), table=OnDevice(i32, 6, 5), length=OnDevice(i32, 6),
             holders=OnDevice(i32, 20))
    v.update(kw)
    return td.Cache(**v)


def test_binding_checks_a_caches_tensors(td, monkeypatch):
    import torch
    i32, bf16, f32 = torch.int32, torch.bfloat16, torch.float32
    some_cache(td, monkeypatch)
    turned = dict(strides=(20 * 4096, 4096, 64, 1024, 1))
    some_cache(td, monkeypatch, keys=OnDevice(bf16, 2, 20, 16, 4, 64, **turned), values=OnDevice(bf16, 2, 20, 16, 4, 64, **turned))
    some_cache(td, monkeypatch, keys=None, values=None, page_size=16)
    for bad in (dict(keys=None), dict(keys=None, values=None), dict(page_size=8), dict(holders=OnDevice(i32, 21)), dict(table=OnDevice(i32, 30)),
                dict(length=OnDevice(i32, 5)), dict(table=OnDevice(f32, 6, 5)), dict(table=OnDevice(i32, 6, 5, device=1)),
                dict(values=OnDevice(f32, 2, 20, 16, 4, 64)), dict(values=OnDevice(bf16, 2, 20, 16, 4, 64, **turned)),
                dict(values=OnDevice(bf16, 2, 20, 16, 4, 64, device=1)), dict(keys=OnDevice(i32, 2, 20, 16, 4, 64), values=OnDevice(i32, 2, 20, 16, 4, 64)),
                dict(keys=OnDevice(bf16, 2, 20, 16, 4, 64, strides=(0, 4096, 256, 64, 1)), values=OnDevice(bf16, 2, 20, 16, 4, 64, strides=(0, 4096, 256, 64, 1))),
                dict(holders=OnDevice(i32, 20, device=-1))):
        with pytest.raises(ValueError):
            some_cache(td, monkeypatch, **bad)


def test_binding_checks_the_calls_tensors(td, monkeypatch):
    import torch
    i32, bf16, f32 = torch.int32, torch.bfloat16, torch.float32
    c = some_cache(td, monkeypatch)
    out = td.AttentionBuffers(3, 8, 64, bf16, out=OnDevice(bf16, 3, 8, 64))
    q, kv, cu = OnDevice(bf16, 3, 8, 64), OnDevice(bf16, 3, 4, 64), OnDevice(i32, 7)
    for call in (lambda: td.cache_extend(c, OnDevice(i32, 5), stream=0), lambda: td.cache_extend(c, OnDevice(torch.int64, 6), stream=0),
                 lambda: td.cache_extend(c, None, OnDevice(i32, 6), stream=0), lambda: td.cache_fork(c, OnDevice(i32, 6, device=1), stream=0),
                 lambda: td.cache_free(c, OnDevice(i32, 6), stream=0), lambda: td.cache_compact(c, OnDevice(i32, 1), OnDevice(i32, 19), stream=0),
                 lambda: td.cache_write(c, kv, OnDevice(bf16, 2, 4, 64), cu, stream=0), lambda: td.cache_write(c, q, q, cu, stream=0),
                 lambda: td.cache_write(c, kv, kv, OnDevice(i32, 6), stream=0), lambda: td.cache_write(c, OnDevice(f32, 3, 4, 64), OnDevice(f32, 3, 4, 64), cu, stream=0),
                 lambda: td.cache_attention(out, c, OnDevice(bf16, 4, 8, 64), stream=0), lambda: td.cache_attention(out, c, kv, stream=0),
                 lambda: td.cache_attention(out, c, OnDevice(f32, 3, 8, 64), stream=0), lambda: td.cache_attention(out, c, q, OnDevice(i32, 2), stream=0),
                 lambda: td.cache_attention(out, c, OnDevice(bf16, 3, 8, 64, strides=(512, 1, 8)), stream=0),
                 lambda: td.cache_attention(out, c, OnDevice(bf16, 3, 8, 64, device=1), stream=0),
                 lambda: td.AttentionBuffers(3, 8, 64, bf16, out=OnDevice(bf16, 3, 8, 32))):
        with pytest.raises(ValueError):
            call()


def test_cache_kernels_do_not_read_through_the_read_only_path():
    csrc = os.path.join(ROOT, "paper_2507_19017_b200", "csrc")
    for name in ("td_cache.cu", "td_cache.cuh", "td_attend.cuh"):
        with open(os.path.join(csrc, name)) as f:
            code = "\n".join(line.split("//")[0] for line in f)
        assert "__ldg" not in code and "global.nc" not in code and "tex." not in code, name
