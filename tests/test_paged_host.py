"""What the paged cache's calls refuse.  The checks come before anything touches a device, so they run without one; the
pointers are numbers that nothing follows."""
import ctypes as C

import pytest

import paper_2510_11958_b200 as pkg
from paper_2510_11958_b200.binding import PAGED_ATTENTION_SCRATCH_BYTES, STATUS, _PagedCache

A = 1 << 20                       # an address, 16-byte aligned


@pytest.fixture(scope="module")
def dll():
    import __graft_entry__
    __graft_entry__.build()
    return pkg.load_library()


def _cache(**kw):
    c = dict(k=A, v=A, dtype=1, n_pages=100, page_size=16, n_kv_heads=2, head_dim=128, page_stride=4096, head_stride=2048, row_stride=128)
    c.update(kw)
    return C.byref(_PagedCache(*(c[n] for n, _ in _PagedCache._fields_)))


def _plan(dll, **kw):
    a = dict(lens=A, n_new=A, n_requests=4, page_size=16, table=A, table_stride=10, free_pages=A, n_pages=100, n_free=A, n_rows=8, row_start=A,
             position=A, slot=A, granted=A, lens_out=A, n_free_out=A, stream=None)
    a.update(kw)
    return dll.dmtd_paged_plan(*a.values())


def _append(dll, cache=None, **kw):
    a = dict(q=A, k=A, v=A, dtype=0, q_stride=1024, k_stride=256, v_stride=256, n_rows=8, nq=8, q_norm=None, k_norm=None, eps=1e-6, theta=1e6,
             position=A, slot=A, cache=cache or _cache(), q_out=A, stream=None)
    a.update(kw)
    return dll.dmtd_paged_append(*a.values())


def _attention(dll, cache=None, **kw):
    a = dict(q=A, q_dtype=1, q_stride=1024, n_rows=8, nq=8, row_start=A, lens=A, n_requests=4, table=A, table_stride=10, max_new=0,
             cache=cache or _cache(), scratch=A, scratch_bytes=PAGED_ATTENTION_SCRATCH_BYTES, out=2 * A, stream=None)
    a.update(kw)
    return dll.dmtd_paged_attention(*a.values())


@pytest.mark.parametrize("want,kw", [
    ("INVALID_ARG", dict(n_requests=-1)), ("INVALID_ARG", dict(n_rows=-1)), ("INVALID_ARG", dict(n_pages=0)), ("INVALID_ARG", dict(table_stride=0)),
    ("INVALID_ARG", dict(lens=None)), ("INVALID_ARG", dict(table=None)), ("INVALID_ARG", dict(slot=None)), ("INVALID_ARG", dict(n_free_out=None)),
    ("SHAPE", dict(page_size=12)), ("SHAPE", dict(page_size=0)), ("SHAPE", dict(page_size=-16)),
    ("CAPACITY", dict(n_requests=8193)), ("CAPACITY", dict(n_pages=1 << 27)), ("CAPACITY", dict(n_rows=1 << 30)),
    ("CAPACITY", dict(n_requests=8192, table_stride=1 << 17)),
])
def test_plan_refusals(dll, want, kw):
    assert _plan(dll, **kw) == STATUS[want]
    assert b"paged_plan" in dll.dmtd_last_error(None)


_BAD_CACHES = [
    ("INVALID_ARG", dict(k=None)), ("INVALID_ARG", dict(n_pages=0)), ("SHAPE", dict(dtype=3)), ("SHAPE", dict(head_dim=96)),
    ("SHAPE", dict(n_kv_heads=0)), ("SHAPE", dict(page_size=24)), ("CAPACITY", dict(n_pages=1 << 27)),
    ("INVALID_ARG", dict(row_stride=64)), ("INVALID_ARG", dict(head_stride=-2048)), ("INVALID_ARG", dict(page_stride=4097)),
    ("INVALID_ARG", dict(v=A + 8)),
]


@pytest.mark.parametrize("want,kw", _BAD_CACHES)
def test_cache_refusals(dll, want, kw):
    assert _append(dll, _cache(**kw)) == STATUS[want]
    assert _attention(dll, _cache(**kw)) == STATUS[want]


@pytest.mark.parametrize("want,kw", [
    ("INVALID_ARG", dict(n_rows=-1)), ("SHAPE", dict(dtype=7)), ("INVALID_ARG", dict(q=None)), ("INVALID_ARG", dict(slot=None)),
    ("INVALID_ARG", dict(q_out=None)), ("INVALID_ARG", dict(theta=-1.0)), ("INVALID_ARG", dict(theta=float("nan"))),
    ("INVALID_ARG", dict(theta=float("inf"))), ("INVALID_ARG", dict(eps=-1.0)), ("INVALID_ARG", dict(q_stride=1000)),
    ("INVALID_ARG", dict(k_stride=258)), ("INVALID_ARG", dict(v=A + 4)), ("INVALID_ARG", dict(q_norm=A + 4)), ("INVALID_ARG", dict(k_norm=A + 8)),
    ("INVALID_ARG", dict(q_stride=1032)), ("CAPACITY", dict(nq=65537)),
])
def test_append_refusals(dll, want, kw):
    assert _append(dll, **kw) == STATUS[want]
    assert b"paged_append" in dll.dmtd_last_error(None)


@pytest.mark.parametrize("want,kw", [
    ("INVALID_ARG", dict(n_rows=-1)), ("INVALID_ARG", dict(max_new=-1)), ("INVALID_ARG", dict(table_stride=0)), ("SHAPE", dict(q_dtype=9)),
    ("UNSUPPORTED", dict(q_dtype=2)), ("SHAPE", dict(nq=7)), ("SHAPE", dict(nq=34)), ("CAPACITY", dict(n_requests=8193)),
    ("CAPACITY", dict(n_rows=1 << 22)), ("CAPACITY", dict(table_stride=1 << 27)), ("CAPACITY", dict(scratch_bytes=PAGED_ATTENTION_SCRATCH_BYTES - 1)),
    ("INVALID_ARG", dict(scratch=None)), ("INVALID_ARG", dict(out=None)), ("INVALID_ARG", dict(lens=None)), ("INVALID_ARG", dict(q_stride=1016)),
    ("INVALID_ARG", dict(q_stride=1028)), ("INVALID_ARG", dict(q=A + 2)), ("INVALID_ARG", dict(out=A + 8)), ("INVALID_ARG", dict(scratch=A + 4)),
    ("INVALID_ARG", dict(out=A)),
])
def test_attention_refusals(dll, want, kw):
    assert _attention(dll, **kw) == STATUS[want]
    assert b"paged_attention" in dll.dmtd_last_error(None)


def test_nothing_to_do(dll):
    assert _append(dll, n_rows=0) == 0
    assert _attention(dll, n_rows=0) == 0
    assert _attention(dll, n_requests=0) == 0


def test_the_header_and_the_binding_agree(dll):
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dmtd.h")).read()
    assert eval(re.search(r"DMTD_PAGED_ATTENTION_SCRATCH_BYTES \((.*)\)", text).group(1).replace("u", "")) == PAGED_ATTENTION_SCRATCH_BYTES
    fields = re.search(r"typedef struct \{([^}]*)\} dmtd_paged_cache;", re.sub(r"/\*.*?\*/", "", text, flags=re.S)).group(1)
    names = [n.strip(" *\n") for part in fields.split(";") for n in re.sub(r"^\s*(void|int32_t|int64_t)\s", "", part).split(",")]
    assert [n for n in names if n] == [n for n, _ in _PagedCache._fields_]


def test_tensors_off_the_device_are_refused(dll):
    """Argument marshalling: CPU tensors, wrong counts of arguments (what needs CUDA tensors is tested on a GPU)."""
    import torch
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="table is not on the current CUDA device"):
        pkg.paged_plan(i, i, torch.zeros(2, 3, dtype=torch.int32), i, i[:1], 16, 4, out=[i] * 6)
    k = torch.zeros(3, 2, 16, 64)
    with pytest.raises(ValueError, match="k_cache is not on the current CUDA device"):
        pkg.paged_append(None, k[0], k[0], i, i, k, k)
    with pytest.raises(ValueError, match="k_cache is not"):
        pkg.paged_attention(k[0], i, i, i[None], k, k, scratch=i, out=k[0])
    from paper_2510_11958_b200 import binding
    with pytest.raises(TypeError, match="13 wanted"):
        binding._paged().plan(i)
    with pytest.raises(ValueError, match="is no tensor"):
        binding._paged().attention(*[None] * 9)


def test_the_binding_is_built_anew_for_another_torch(dll, monkeypatch):
    import torch
    from paper_2510_11958_b200 import binding, build
    assert not build._binding_stale()
    assert torch.__version__ in binding._paged().__doc__
    monkeypatch.setattr(torch, "__version__", torch.__version__ + "1")
    assert build._binding_stale()
