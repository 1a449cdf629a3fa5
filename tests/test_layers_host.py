"""CPU tests of the layers' C ABI: exports, refusals before any launch,
workspace sizes, the header as C99, and no register spills in any kernel."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_29119_amd import layers
from paper_2609_29119_amd import nsgcqt as nb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20    # a device address that is never read: every call below is refused, or has nothing to do


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(nb.LIB_PATH):
        pytest.fail("libnsgcqt.so is not built; run python -m paper_2609_29119_amd.build")
    return layers._lib()


def test_every_declared_symbol_is_exported(L):
    text = open(os.path.join(ROOT, "include", "nsgcqt_layers.h")).read()
    names = sorted(set(re.findall(r"^\s*(?:int|int64_t)\s+(nsgcqt_\w+)\s*\(", text, re.M)))
    assert names == sorted(layers.EXPORTS)
    for n in names:
        assert hasattr(L, n), n


class Rows(ctypes.Structure):
    _fields_ = [("offsets", ctypes.c_void_p), ("n_bands", ctypes.c_int64), ("batch", ctypes.c_int64),
                ("rows", ctypes.c_int64)]


class View(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("row", ctypes.c_int64),
                ("head", ctypes.c_int64)]


class Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("n_heads", "n_kv_heads", "head_dim", "left", "right", "sinks")] + [
        ("scale", ctypes.c_double), ("keep", ctypes.c_void_p), ("keep_batch", ctypes.c_int64)]


def ref(x):
    return ctypes.byref(x)


def rows(offsets=FAKE, bands=2, batch=1, n=8):
    return Rows(offsets, bands, batch, n)


def view(data=FAKE, batch=64, row=8, head=8):
    return View(data, batch, row, head)


def shape(heads=2, kv=1, dim=8, left=3, right=0, sinks=0, scale=1.0):
    return Shape(heads, kv, dim, left, right, sinks, scale, None, 0)


def refused(status, code, word):
    assert status == code
    assert word in nb.lib().nsgcqt_last_error().decode()


def test_linear_refusals(L):
    v = view()
    call = lambda dtype=0, r=rows(), x=v, w=FAKE, b=None, y=v, k=8, m=8: L.nsgcqt_band_linear(  # noqa: E731
        dtype, r if r is None else ref(r), x if x is None else ref(x), w, b, y if y is None else ref(y), k, m, None)
    refused(call(dtype=3), nb.EINVAL, "data type")
    refused(call(r=None), nb.EINVAL, "rows is NULL")
    refused(call(r=rows(offsets=None)), nb.EINVAL, "offsets")
    refused(call(r=rows(offsets=FAKE + 4)), nb.EINVAL, "aligned")
    refused(call(r=rows(bands=-1)), nb.EINVAL, "negative")
    refused(call(r=rows(n=1 << 30)), nb.EUNSUPPORTED, "range")
    refused(call(x=None), nb.EINVAL, "x is NULL")
    refused(call(x=view(data=None)), nb.EINVAL, "NULL pointer")
    refused(call(x=view(data=FAKE + 2)), nb.EINVAL, "aligned")
    refused(call(y=view(row=-8)), nb.EINVAL, "negative stride")
    refused(call(w=None), nb.EINVAL, "w is NULL")
    refused(call(k=-1), nb.EINVAL, "width")
    refused(call(m=65537), nb.EUNSUPPORTED, "65,536")
    assert call(r=rows(n=0), w=FAKE) == nb.OK and call(r=rows(batch=0)) == nb.OK
    g = lambda ws, n, dw=FAKE: L.nsgcqt_band_linear_grad_weight(0, ref(rows()), ref(v), ref(v), dw, None, 8, 8, ws, n, None)  # noqa: E731
    refused(g(FAKE, 16), nb.EWORKSPACE, "required")
    refused(g(None, 1 << 30), nb.EINVAL, "workspace")
    refused(g(FAKE, 1 << 30, dw=None), nb.EINVAL, "dw is NULL")
    assert L.nsgcqt_band_linear_workspace(2, 1, 8, -1, 8) == nb.EINVAL
    assert L.nsgcqt_band_linear_workspace(2, 1, 8, 8, 8) >= 4 * 2 * 72


def test_attention_refusals(L):
    v = view()
    call = lambda dtype=0, r=rows(), s=shape(), q=v, k=v: L.nsgcqt_band_attention(  # noqa: E731
        dtype, ref(r), s if s is None else ref(s), ref(q), ref(k), ref(v), ref(v), None, None)
    refused(call(dtype=-1), nb.EINVAL, "data type")
    refused(call(s=None), nb.EINVAL, "shape is NULL")
    refused(call(s=shape(heads=3, kv=2)), nb.EINVAL, "divide")
    refused(call(s=shape(kv=0)), nb.EINVAL, "divide")
    refused(call(s=shape(dim=0)), nb.EINVAL, "head_dim")
    refused(call(s=shape(dim=129)), nb.EUNSUPPORTED, "128")
    refused(call(s=shape(left=-1)), nb.EINVAL, "negative")
    for bad in (0.0, -1.0, float("inf"), float("nan"), 1e300, 1e-300):
        refused(call(s=shape(scale=bad)), nb.EINVAL, "scale")
    refused(call(q=view(data=FAKE + 1)), nb.EINVAL, "aligned")
    assert call(r=rows(n=0)) == nb.OK
    grad = lambda stats, ws, n: L.nsgcqt_band_attention_grad(  # noqa: E731
        0, ref(rows()), ref(shape()), *[ref(v)] * 4, stats, *[ref(v)] * 4, ws, n, None)
    refused(grad(None, FAKE, 1 << 30), nb.EINVAL, "stats")
    refused(grad(FAKE, FAKE, 8), nb.EWORKSPACE, "required")
    refused(grad(FAKE, FAKE + 4, 1 << 30), nb.EINVAL, "workspace")
    few = L.nsgcqt_band_attention_workspace(ref(rows(n=4000)), ref(shape()))
    more = L.nsgcqt_band_attention_workspace(ref(rows(n=4000)), ref(shape(sinks=4)))
    assert 4 * 2 * 4000 <= few < more


def test_rotary_refusals(L):
    v, sec = view(), (ctypes.c_int32 * 4)(1, 1, 1, 1)
    call = lambda q=v, heads=1, dim=8, pos=FAKE, kind=1, sections=sec, axes=2, freqs=FAKE: L.nsgcqt_rotary(  # noqa: E731
        0, ref(q), ref(v), heads, None, None, 0, 1, 8, dim, pos, kind, 8, 0, freqs, sections, axes, 0, 0, None)
    refused(call(axes=0), nb.EINVAL, "n_axes")
    refused(call(axes=5), nb.EINVAL, "n_axes")
    refused(call(sections=None), nb.EINVAL, "sections")
    refused(call(dim=3), nb.EINVAL, "pairs")
    refused(call(sections=(ctypes.c_int32 * 4)(2, -1, 0, 0)), nb.EINVAL, "negative")
    refused(call(kind=3), nb.EINVAL, "positions")
    refused(call(pos=FAKE + 4), nb.EINVAL, "positions")
    refused(call(pos=None), nb.EINVAL, "positions")
    refused(call(freqs=None), nb.EINVAL, "freqs")
    refused(call(heads=-1), nb.EINVAL, "negative")
    refused(call(q=view(data=FAKE + 2)), nb.EINVAL, "aligned")
    assert call(heads=0) == nb.OK


def test_step_and_fill_refusals(L):
    v = view()
    call = lambda n=2, heads=2, kv=1, dim=8, window=8, sinks=0, scale=1.0, kc=FAKE, pos=FAKE, ws=FAKE, nws=1 << 40: (  # noqa: E731
        L.nsgcqt_attention_step(0, n, heads, kv, dim, window, sinks, scale, *[ref(v)] * 4, kc, FAKE, pos, ws, nws, None))
    refused(call(n=-1), nb.EINVAL, "n_streams")
    refused(call(heads=3, kv=2), nb.EINVAL, "divide")
    refused(call(dim=200), nb.EUNSUPPORTED, "128")
    refused(call(window=0), nb.EINVAL, "window")
    refused(call(sinks=-1), nb.EINVAL, "sinks")
    refused(call(window=1 << 30), nb.EUNSUPPORTED, "range")
    refused(call(scale=0.0), nb.EINVAL, "scale")
    refused(call(kc=None), nb.EINVAL, "cache")
    refused(call(pos=FAKE + 4), nb.EINVAL, "pos")
    refused(call(window=100000, nws=16), nb.EWORKSPACE, "required")
    refused(call(window=100000, ws=None), nb.EINVAL, "workspace")
    assert call(n=0) == nb.OK
    fill = lambda r=rows(), window=4, kc=FAKE: L.nsgcqt_cache_fill(  # noqa: E731
        0, ref(r), 1, 8, window, 0, ref(v), ref(v), kc, FAKE, None)
    refused(fill(window=0), nb.EINVAL, "window")
    refused(fill(kc=None), nb.EINVAL, "cache")
    refused(fill(r=rows(bands=70000)), nb.EUNSUPPORTED, "streams")
    assert fill(r=rows(n=0)) == nb.OK


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not available")
def test_header_is_c99(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "nsgcqt_layers.h"\n'
                   "int main(void) { nsgcqt_view v = {0}; (void)v;\n"
                   "  return nsgcqt_band_linear_workspace(2, 1, 8, -1, 8) == NSGCQT_EINVAL ? 0 : 1; }\n")
    lib = os.path.dirname(nb.LIB_PATH)
    exe = tmp_path / "use"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe),
                    "-L", lib, "-lnsgcqt", "-Wl,-rpath," + lib], check=True, capture_output=True)
    assert subprocess.run([str(exe)], timeout=60).returncode == 0


@pytest.mark.parametrize("name", ["linear", "rotary", "attention", "attention_grad", "step"])
def test_no_kernel_spills(name, tmp_path):
    from paper_2609_29119_amd.build import LAYER_FLAGS, LAYERS
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    assert name in LAYERS
    r = subprocess.run([hipcc, *LAYER_FLAGS, "--cuda-device-only", "-c",
                        os.path.join(ROOT, "paper_2609_29119_amd", "csrc", "layers", f"{name}.hip"),
                        "-o", str(tmp_path / "dev.o"), "-Rpass-analysis=kernel-resource-usage"],
                       capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stderr[-2000:]
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    scratch = [int(v) for v in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)]
    assert names and len(names) == len(scratch)
    assert not [(n, s) for n, s in zip(names, scratch) if s]


def run_on_the_host(name, tmp_path, *args):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = tmp_path / name
    subprocess.run([hipcc, "-x", "hip", "--offload-host-only", "-O2", "-fwrapv", "-std=c++17", "-w",
                    os.path.join(ROOT, "tests", "c", name + ".cpp"), "-o", str(exe)], check=True, timeout=300)
    r = subprocess.run([str(exe), *args], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout


@pytest.mark.parametrize("seed", [0, 1])
def test_band_search(seed, tmp_path):
    """The search for a work item's band against a plain scan, on the host: 0 to 20,000 bands, among them those where
    its last round goes in steps of more than one; offsets in any order keep every tile and chunk in range."""
    run_on_the_host("band_search", tmp_path, str(seed))


def test_attention_range_of_the_longest_rows(tmp_path):
    """The end of a key tile's queries, with a window as long as the longest row."""
    run_on_the_host("attention_range", tmp_path)


def test_sizes_past_what_a_launch_takes(L):
    """Sizes that one launch cannot take are refused as such before anything is launched, also where their product
    passes 64 bits; so are workspaces."""
    v = view()
    step = lambda n, heads, kv: L.nsgcqt_attention_step(  # noqa: E731
        0, n, heads, kv, 8, 8, 0, 1.0, *[ref(v)] * 4, FAKE, FAKE, FAKE, None, 0, None)
    refused(step(1 << 22, 4, 4), nb.EUNSUPPORTED, "workgroups")        # 2^24 workgroups of 256 threads
    refused(step(1 << 20, 16, 1), nb.EUNSUPPORTED, "workgroups")       # outputs
    attend = lambda r, s: L.nsgcqt_band_attention(0, ref(r), ref(s), *[ref(v)] * 4, None, None)  # noqa: E731
    refused(attend(rows(bands=1 << 20, batch=16, n=1 << 20), shape(heads=8, kv=2)), nb.EUNSUPPORTED, "workgroups")
    # 2^24 tiles of 2^30 signals and 2^16 heads: the product is 0 in 64 bits
    wraps = rows(bands=(1 << 24) - 2 - 8, batch=1 << 30, n=1024)
    refused(attend(wraps, shape(heads=65536, kv=65536)), nb.EUNSUPPORTED, "workgroups")
    refused(L.nsgcqt_band_attention_workspace(ref(rows(bands=(1 << 24) - 4, batch=1 << 30, n=1024)),
                                              ref(shape(heads=65536, kv=65536, sinks=4))), nb.EUNSUPPORTED, "workspace")
    refused(L.nsgcqt_band_attention_grad(0, ref(rows(bands=1 << 20, batch=16, n=1 << 20)), ref(shape(heads=8, kv=8)),
                                         *[ref(v)] * 4, FAKE, *[ref(v)] * 4, FAKE, 1 << 60, None),
            nb.EUNSUPPORTED, "workgroups")
    refused(L.nsgcqt_band_linear(0, ref(rows(bands=1 << 24, batch=1, n=1024)), ref(v), FAKE, None, ref(v), 8, 8, None),
            nb.EUNSUPPORTED, "workgroups")
    refused(L.nsgcqt_rotary(0, ref(v), ref(v), 1, None, None, 0, 1 << 20, 1 << 10, 64, FAKE, 1, 8, 0, FAKE,
                            (ctypes.c_int32 * 4)(32, 0, 0, 0), 1, 0, 0, None), nb.EUNSUPPORTED, "workgroups")
    # 2^34 tiles of 2^32 weights, 4 bytes each: 0 in 64 bits
    n = L.nsgcqt_band_linear_workspace(2, 1 << 30, 1 << 10, 65536, 65535)
    refused(n, nb.EUNSUPPORTED, "workspace")
    refused(L.nsgcqt_band_linear_grad_weight(0, ref(rows(batch=1 << 30, n=1 << 10)), ref(v), ref(v), FAKE, FAKE, 65536,
                                             65535, FAKE, 1 << 60, None), nb.EUNSUPPORTED, "workspace")


def test_gradient_workspace_with_many_sinks(L):
    """The partial sums of the sinks are bounded: 131,072 tokens, every one a sink, 2 kv heads of 128."""
    s, r = shape(heads=8, kv=2, dim=128, left=1023, sinks=131072), rows(bands=1, n=131072)
    assert L.nsgcqt_band_attention_workspace(ref(r), ref(s)) <= 4 * 131072 * 8 + 2 * (2 * 2 * 131072 * 2 * 128) * 1.05


def test_strides_of_axes_of_one_element_are_not_read(L):
    """What is not read may hold anything: both calls below are refused for their workspace, later than for strides."""
    v = view(row=-(1 << 62))
    refused(L.nsgcqt_attention_step(0, 2, 2, 1, 8, 100000, 0, 1.0, *[ref(v)] * 4, FAKE, FAKE, FAKE, FAKE, 16, None),
            nb.EWORKSPACE, "required")
    v = view(batch=-3, head=-5)
    refused(L.nsgcqt_band_linear_grad_weight(0, ref(rows(batch=1)), ref(v), ref(v), FAKE, None, 8, 8, FAKE, 16, None),
            nb.EWORKSPACE, "required")
    v = view(batch=-3)
    refused(L.nsgcqt_band_linear_grad_weight(0, ref(rows(batch=2)), ref(v), ref(v), FAKE, None, 8, 8, FAKE, 16, None),
            nb.EINVAL, "negative stride")
