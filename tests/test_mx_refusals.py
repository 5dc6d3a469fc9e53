"""What the operators on microscaled tensors, norms and caches refuse (CPU: every refusal comes before any CUDA call)."""
import ctypes
import re

import pytest

from paper_1805_07941_b200 import binding

A = 1 << 20                                                 # stands for an aligned device address


@pytest.fixture(scope="module")
def lib():
    binding.build_library()
    return binding.lib()


@pytest.mark.parametrize("name", ["qmx_linear_desc", "qrmsnorm_args", "qcache_desc", "qcache_values"])
def test_structs_match_the_header(name):
    text = re.sub(r"/\*.*?\*/", "", open(binding.HEADER_PATH).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text).group(1)
    fields = []
    for decl in body.split(";"):
        names = re.sub(r"^\s*(const\s+)?(void|int|long long|double|uint8_t)\b", "", decl)
        fields += [n.strip(" *\n") for n in names.split(",") if n.strip()]
    assert fields == [n for n, _ in getattr(binding, name)._fields_]


def test_structs_as_bytes_have_the_structures_layout():
    for packed, structure in ((binding._NORM_ARGS, binding.qrmsnorm_args), (binding._CACHE_VALUES, binding.qcache_values)):
        names = [n for n, _ in structure._fields_]
        assert packed.size == ctypes.sizeof(structure)
        s = structure.from_buffer_copy(packed.pack(*range(1, len(names) + 1)))
        assert [int(getattr(s, n)) for n in names] == list(range(1, len(names) + 1))


def test_sizes(lib):
    assert lib.qmx_code_bytes(3, 33) == 3 * 32 and lib.qmx_scale_bytes(3, 33, 0) == 6
    assert lib.qmx_scale_bytes(129, 129, 1) == 2 * 2 * 512
    assert lib.qmx_code_bytes(0, 5) == 0 and lib.qmx_scale_bytes(4, 0, 0) == 0 and lib.qmx_scale_bytes(4, 4, 2) == 0
    assert lib.qmx_code_bytes(1 << 33, 64) == 1 << 38


@pytest.mark.parametrize("change,code", [
    (dict(x=None), "BAD_ARG"), (dict(codes=None), "BAD_ARG"), (dict(scales=None), "BAD_ARG"), (dict(type=3), "BAD_ARG"),
    (dict(rows=0), "BAD_ARG"), (dict(rows=-1), "BAD_ARG"), (dict(K=0), "BAD_ARG"), (dict(ld=63), "BAD_ARG"),
    (dict(rule=2), "BAD_ARG"), (dict(layout=2), "BAD_ARG"), (dict(codes=A + 8), "ALIGNMENT"), (dict(scales=A + 4), "ALIGNMENT"),
    (dict(x=A + 2), "ALIGNMENT"), (dict(rows=1 << 31, K=64), "UNSUPPORTED_SHAPE"), (dict(K=(1 << 28) + 1, ld=1 << 29), "UNSUPPORTED_SHAPE"),
    (dict(ld=(1 << 40) + 1), "UNSUPPORTED_SHAPE")])
def test_codec(lib, change, code):
    a = dict(x=A, type=0, rows=4, K=64, ld=64, rule=0, layout=1, codes=A, scales=A)
    a.update(change)
    assert lib.qmx_quantize(a["x"], a["type"], a["rows"], a["K"], a["ld"], a["rule"], a["layout"], a["codes"], a["scales"], None) == \
        getattr(binding, "ERR_" + code)
    if "rule" not in change:
        assert lib.qmx_dequantize(a["codes"], a["scales"], a["rows"], a["K"], a["layout"], a["x"], a["type"], a["ld"], None) == \
            getattr(binding, "ERR_" + code)


@pytest.mark.parametrize("change,code", [
    (dict(w=None), "BAD_ARG"), (dict(s=None), "BAD_ARG"), (dict(N=0), "BAD_ARG"), (dict(K=-4), "BAD_ARG"), (dict(type=7), "BAD_ARG"),
    (dict(w=A + 8), "ALIGNMENT"), (dict(s=A + 8), "ALIGNMENT"), (dict(bias=A + 2), "ALIGNMENT"), (dict(K=(1 << 28) + 1), "UNSUPPORTED_SHAPE")])
def test_linear_create(lib, change, code):
    a = dict(w=A, s=A, bias=None, N=64, K=64, type=0)
    a.update(change)
    h = ctypes.c_void_p(5)
    d = binding.qmx_linear_desc(N=a["N"], K=a["K"], relu=0, type=a["type"])
    assert lib.qmx_linear_create(ctypes.byref(h), ctypes.byref(d), a["w"], a["s"], a["bias"]) == getattr(binding, "ERR_" + code)
    assert not h.value
    assert lib.qmx_linear_create(None, ctypes.byref(d), a["w"], a["s"], a["bias"]) == binding.ERR_BAD_ARG


def test_linear_without_a_handle(lib):
    buf = ctypes.create_string_buffer(10)
    assert lib.qmx_linear_run(None, A, A, 1, A, 64, None) == binding.ERR_BAD_ARG
    assert lib.qmx_linear_status(None) == binding.ERR_BAD_ARG and lib.qmx_linear_destroy(None) == binding.ERR_BAD_ARG
    assert lib.qmx_linear_set_wait_limit(None, 1) == binding.ERR_BAD_ARG and lib.qmx_linear_describe(None, buf, 10) == binding.ERR_BAD_ARG


@pytest.mark.parametrize("change,code", [
    (dict(d_x=None), "BAD_ARG"), (dict(d_gain=None), "BAD_ARG"), (dict(d_codes=None), "BAD_ARG"), (dict(out=1, d_scales=None), "BAD_ARG"),
    (dict(out=3), "BAD_ARG"), (dict(type=-1), "BAD_ARG"), (dict(C=0), "BAD_ARG"), (dict(rows=0), "BAD_ARG"), (dict(ld_x=10), "BAD_ARG"),
    (dict(eps=-1e-6), "BAD_ARG"), (dict(eps=float("nan")), "BAD_ARG"), (dict(eps=float("inf")), "BAD_ARG"), (dict(e=127), "BAD_ARG"),
    (dict(e=-127), "BAD_ARG"), (dict(d_residual=A, ld_residual=63), "BAD_ARG"), (dict(d_sum=A, ld_sum=63), "BAD_ARG"),
    (dict(d_sum=A, ld_sum=72), "BAD_ARG"), (dict(d_sum=3 * A, d_residual=3 * A, ld_residual=64, ld_sum=65), "BAD_ARG"),
    (dict(d_x=A + 1), "ALIGNMENT"), (dict(d_gain=A + 1), "ALIGNMENT"), (dict(d_sum=2 * A + 1, ld_sum=64), "ALIGNMENT"),
    (dict(out=2, layout=2), "BAD_ARG"), (dict(out=2, d_codes=A + 4), "ALIGNMENT"), (dict(out=2, d_scales=A + 4), "ALIGNMENT"),
    (dict(C=(1 << 24) + 1, ld_x=1 << 25), "UNSUPPORTED_SHAPE"), (dict(rows=1 << 31), "UNSUPPORTED_SHAPE")])
def test_norm(lib, change, code):
    a = dict(d_x=A, d_gain=A, type=1, C=64, rows=2, ld_x=64, eps=1e-6, out=0, e=0, layout=1, d_codes=A, d_scales=A)
    a.update(change)
    args = binding.qrmsnorm_args(**a)
    assert lib.qrmsnorm(ctypes.byref(args), None) == getattr(binding, "ERR_" + code)
    assert lib.qrmsnorm(None, None) == binding.ERR_BAD_ARG


@pytest.mark.parametrize("change,code", [
    (dict(format=2), "BAD_ARG"), (dict(heads=0), "BAD_ARG"), (dict(D=0), "BAD_ARG"), (dict(num_slots=0), "BAD_ARG"), (dict(rows=-1), "BAD_ARG"),
    (dict(type=3), "BAD_ARG"), (dict(d_k_codes=None), "BAD_ARG"), (dict(d_v_scales=None), "BAD_ARG"), (dict(slots=None), "BAD_ARG"),
    (dict(values=None), "BAD_ARG"), (dict(stride=-1), "BAD_ARG"), (dict(D=1025), "UNSUPPORTED_SHAPE"), (dict(rows=1 << 30), "UNSUPPORTED_SHAPE"),
    (dict(slots=A + 4), "ALIGNMENT"), (dict(values=A + 2), "ALIGNMENT"), (dict(format=1, d_v_codes=A + 8), "ALIGNMENT")])
def test_cache(lib, change, code):
    a = dict(format=0, heads=2, D=64, num_slots=8, d_k_codes=A, d_k_scales=A, d_v_codes=A, d_v_scales=A, rows=3, type=0, slots=A, values=A,
             stride=128)
    a.update(change)
    cache = binding.qcache_desc(a["format"], a["heads"], a["D"], a["num_slots"], a["d_k_codes"], a["d_k_scales"], a["d_v_codes"], a["d_v_scales"])
    v = binding.qcache_values(a["values"], a["stride"], 64)
    want = getattr(binding, "ERR_" + code)
    b = ctypes.byref
    assert lib.qcache_write(b(cache), b(v), b(v), a["type"], a["slots"], a["rows"], None) == want
    assert lib.qcache_read(b(cache), a["slots"], a["rows"], b(v), b(v), a["type"], None) == want
    assert lib.qcache_write(None, b(v), b(v), 0, A, 1, None) == binding.ERR_BAD_ARG
    assert lib.qcache_write(b(cache), None, b(v), 0, A, 1, None) == binding.ERR_BAD_ARG


def test_an_empty_list_of_slots_is_fine(lib):
    cache = binding.qcache_desc(0, 2, 64, 8, A, A, A, A)
    v = binding.qcache_values(A, 128, 64)
    assert lib.qcache_write(ctypes.byref(cache), ctypes.byref(v), ctypes.byref(v), 0, A, 0, None) == binding.QCONV_OK
