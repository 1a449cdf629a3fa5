"""CPU tests of the C ABI of the decayed attention, the group norm and the gated product: refusals before any launch,
workspace sizes, slots of segments, and no register spills in any kernel."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_29119_amd import layers
from paper_2609_29119_amd import nsgcqt as nb
from test_layers_host import FAKE, ROOT, L, ref, refused, rows, run_on_the_host, view  # noqa: F401


class Decay(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("n_heads", "n_kv_heads", "head_dim")] + [
        ("scale", ctypes.c_double), ("log_decay", ctypes.c_void_p), ("keep", ctypes.c_void_p), ("keep_batch", ctypes.c_int64)]


class Norm(ctypes.Structure):
    _fields_ = [("channels", ctypes.c_int64), ("groups", ctypes.c_int64), ("eps", ctypes.c_double), ("w", ctypes.c_void_p),
                ("b", ctypes.c_void_p), ("w_band", ctypes.c_int64), ("b_band", ctypes.c_int64), ("act", ctypes.c_int)]


def decay(heads=2, kv=1, dim=8, scale=1.0, lam=FAKE):
    return Decay(heads, kv, dim, scale, lam, None, 0)


def norm(channels=8, groups=2, eps=1e-5, w=None, b=None, w_band=8, b_band=8, act=0):
    return Norm(channels, groups, eps, w, b, w_band, b_band, act)


def test_packed_structs_are_the_header_s():
    """The binding passes structs as packed bytes; theirs are the C structs' sizes."""
    assert layers._decay_shape and len(layers._decay_shape(1, 1, 1, 1.0, 0, 0, 0)) == ctypes.sizeof(Decay)
    assert len(layers._norm_shape(1, 1, 1.0, 0, 0, 0, 0, 0)) == ctypes.sizeof(Norm)


def test_decay_refusals(L):  # noqa: F811
    v = view()
    call = lambda dtype=0, r=rows(), s=decay(), q=v, state=None, ws=None, n=0: L.nsgcqt_decay_attention(  # noqa: E731
        dtype, ref(r), s if s is None else ref(s), ref(q), ref(v), ref(v), ref(v), state, ws, n, None)
    refused(call(dtype=7), nb.EINVAL, "data type")
    refused(call(s=None), nb.EINVAL, "shape is NULL")
    refused(call(s=decay(heads=3, kv=2)), nb.EINVAL, "divide")
    refused(call(s=decay(kv=0)), nb.EINVAL, "divide")
    refused(call(s=decay(dim=0)), nb.EINVAL, "head_dim")
    refused(call(s=decay(dim=129)), nb.EUNSUPPORTED, "128")
    refused(call(s=decay(heads=65537, kv=1)), nb.EUNSUPPORTED, "65,536")
    for bad in (float("inf"), float("nan"), 1e300):
        refused(call(s=decay(scale=bad)), nb.EINVAL, "scale")
    refused(call(s=decay(lam=None)), nb.EINVAL, "log_decay")
    refused(call(s=decay(lam=FAKE + 2)), nb.EINVAL, "log_decay")
    refused(call(state=FAKE + 2), nb.EINVAL, "state")
    refused(call(q=view(data=FAKE + 1)), nb.EINVAL, "aligned")
    refused(call(r=rows(bands=-1)), nb.EINVAL, "negative")
    refused(call(r=rows(n=100000), n=16, ws=FAKE), nb.EWORKSPACE, "required")
    refused(call(r=rows(n=100000), n=1 << 40), nb.EINVAL, "workspace")
    assert call(r=rows(n=0), s=decay(lam=None)) == nb.OK and call(r=rows(batch=0)) == nb.OK
    grad = lambda r=rows(), s=decay(), dk=v, ws=None, n=0: L.nsgcqt_decay_attention_grad(  # noqa: E731
        0, ref(r), ref(s), *[ref(v)] * 5, ref(dk), ref(v), ws, n, None)
    refused(grad(dk=view(data=None)), nb.EINVAL, "dk has a NULL pointer")
    refused(grad(r=rows(n=100000), n=16, ws=FAKE), nb.EWORKSPACE, "required")
    refused(grad(s=decay(lam=None)), nb.EINVAL, "log_decay")
    assert grad(r=rows(n=0)) == nb.OK
    size = lambda r, s=decay(), g=0: L.nsgcqt_decay_attention_workspace(ref(r), ref(s), g)  # noqa: E731
    assert size(rows(n=64)) == 0 < size(rows(n=4000)) < size(rows(n=4000), g=1)
    # short bands of many signals need none, however many
    assert size(rows(n=300, batch=1 << 20, bands=300), decay(heads=8, kv=8, dim=128)) == 0
    # and a long row a share of its own size: 131,072 tokens, 8 heads of 128
    assert size(rows(n=131072, bands=1), decay(heads=8, kv=8, dim=128)) <= 131072 * 8 * 128 * 2 * 2


def test_decay_step_refusals(L):  # noqa: F811
    v = view()
    call = lambda n=2, heads=2, kv=1, dim=8, scale=1.0, st=FAKE, pos=FAKE, lam=FAKE, o=v: L.nsgcqt_decay_step(  # noqa: E731
        0, n, heads, kv, dim, scale, ref(v), ref(v), ref(v), ref(o), st, pos, lam, None)
    refused(call(n=-1), nb.EINVAL, "n_streams")
    refused(call(heads=3, kv=2), nb.EINVAL, "divide")
    refused(call(dim=200), nb.EUNSUPPORTED, "128")
    refused(call(scale=float("nan")), nb.EINVAL, "scale")
    refused(call(st=None), nb.EINVAL, "state is NULL")
    refused(call(st=FAKE + 1), nb.EINVAL, "state")
    refused(call(pos=FAKE + 4), nb.EINVAL, "pos")
    refused(call(lam=None), nb.EINVAL, "log_decay")
    refused(call(o=view(data=FAKE + 3)), nb.EINVAL, "aligned")
    refused(call(n=1 << 24), nb.EUNSUPPORTED, "workgroups")
    refused(call(n=1 << 62, heads=4, kv=4), nb.EUNSUPPORTED, "workgroups")
    assert call(n=0, st=None) == nb.OK


def test_norm_refusals(L):  # noqa: F811
    v = view()
    call = lambda dtype=0, r=rows(), s=norm(), x=v, st=None, ws=None, n=0: L.nsgcqt_band_norm(  # noqa: E731
        dtype, ref(r), s if s is None else ref(s), ref(x), ref(v), st, ws, n, None)
    refused(call(dtype=3), nb.EINVAL, "data type")
    refused(call(s=None), nb.EINVAL, "shape is NULL")
    refused(call(s=norm(groups=3)), nb.EINVAL, "groups")
    refused(call(s=norm(groups=0)), nb.EINVAL, "groups")
    for bad in (0.0, -1.0, float("nan"), float("inf"), 1e-31):
        refused(call(s=norm(eps=bad)), nb.EINVAL, "eps")
    refused(call(s=norm(act=4)), nb.EINVAL, "activation")
    refused(call(s=norm(act=-1)), nb.EINVAL, "activation")
    refused(call(s=norm(w=FAKE + 2)), nb.EINVAL, "aligned")
    refused(call(s=norm(w=FAKE, w_band=-8)), nb.EINVAL, "stride")
    refused(call(s=norm(channels=4104, groups=1)), nb.EUNSUPPORTED, "4,096")
    refused(call(s=norm(channels=2048, groups=2048)), nb.EUNSUPPORTED, "1,024")
    refused(call(st=FAKE + 8), nb.EINVAL, "stats")
    refused(call(x=view(row=-8)), nb.EINVAL, "negative stride")
    refused(call(r=rows(n=100000), ws=FAKE, n=8), nb.EWORKSPACE, "required")
    assert call(r=rows(n=0)) == nb.OK and call(s=norm(channels=0)) == nb.OK
    grad = lambda st=FAKE, dw=FAKE, ws=FAKE, n=1 << 40, r=rows(): L.nsgcqt_band_norm_grad(  # noqa: E731
        0, ref(r), ref(norm()), ref(v), st, ref(v), ref(v), dw, None, ws, n, None)
    refused(grad(st=None), nb.EINVAL, "stats")
    refused(grad(dw=FAKE + 2), nb.EINVAL, "dw")
    refused(grad(n=8), nb.EWORKSPACE, "required")
    refused(grad(ws=FAKE + 4), nb.EINVAL, "workspace")
    refused(grad(r=rows(bands=1 << 24, batch=1 << 30)), nb.EUNSUPPORTED, "")
    size = lambda r, g=0, w=0: L.nsgcqt_band_norm_workspace(0, ref(r), ref(norm()), g, w)  # noqa: E731
    assert size(rows(n=8)) == 0 < size(rows(n=100000))
    # single tokens of a million signals: what dw and db are made of stays far below the data
    assert size(rows(n=1, batch=1 << 20, bands=1), 1, 1) <= (1 << 20) * 8 * 4 / 4


def test_gated_refusals(L):  # noqa: F811
    v = view()
    call = lambda dtype=0, x=v, w=FAKE, b=None, k=8, m=8, act=1, r=rows(): L.nsgcqt_band_gated(  # noqa: E731
        dtype, ref(r), ref(x), w, b, ref(v), k, m, act, None)
    refused(call(dtype=9), nb.EINVAL, "data type")
    refused(call(w=None), nb.EINVAL, "w is NULL")
    refused(call(w=FAKE + 2), nb.EINVAL, "aligned")
    refused(call(b=FAKE + 1), nb.EINVAL, "bias")
    refused(call(k=-1), nb.EINVAL, "width")
    refused(call(m=32769), nb.EUNSUPPORTED, "32,768")
    refused(call(act=5), nb.EINVAL, "activation")
    refused(call(x=view(data=None)), nb.EINVAL, "NULL pointer")
    refused(call(r=rows(bands=1 << 24, n=1024)), nb.EUNSUPPORTED, "workgroups")
    assert call(r=rows(n=0)) == nb.OK
    grad = lambda dw=FAKE, db=None, ws=FAKE, n=1 << 40, r=rows(): L.nsgcqt_band_gated_grad(  # noqa: E731
        0, ref(r), ref(v), FAKE, None, ref(v), ref(v), dw, db, 8, 8, 1, ws, n, None)
    refused(grad(n=16), nb.EWORKSPACE, "required")
    refused(grad(ws=None), nb.EINVAL, "workspace")
    refused(grad(dw=None, db=FAKE), nb.EINVAL, "db without dw")
    refused(grad(dw=FAKE + 1), nb.EINVAL, "aligned")
    assert L.nsgcqt_band_gated_workspace(ref(rows()), 8, 8) > 0
    refused(L.nsgcqt_band_gated_workspace(ref(rows(batch=1 << 30, n=1 << 10)), 65536, 32768), nb.EUNSUPPORTED, "workspace")


@pytest.mark.parametrize("seed", [0, 1])
def test_segments_have_slots_of_their_own(seed, tmp_path):
    run_on_the_host("segment_slots", tmp_path, str(seed))


@pytest.mark.parametrize("name", ["decay", "norm", "gated"])
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


def test_gated_gradients_of_more_workgroups_than_a_launch_takes(L):  # noqa: F811
    """The weights' gradient has workgroups of 512: half as many as the other kernels' fit a launch."""
    v = view()
    grad = lambda bands: L.nsgcqt_band_gated_grad(  # noqa: E731
        0, ref(rows(n=8, bands=bands)), ref(v), FAKE, None, ref(v), None, FAKE, None, 8, 8, 1, FAKE, 1 << 40, None)
    refused(grad(9_000_000), nb.EUNSUPPORTED, "8388607 workgroups")
    refused(grad(1 << 24), nb.EUNSUPPORTED, "workgroups")


def test_norms_of_more_workgroups_than_launches_take(L):  # noqa: F811
    v = view()
    call = lambda r, s=norm(): L.nsgcqt_band_norm(0, ref(r), ref(s), ref(v), ref(v), None, None, 0, None)  # noqa: E731
    refused(call(rows(n=8, bands=1 << 23, batch=1 << 12)), nb.EUNSUPPORTED, "2^34")
    refused(call(rows(n=1, bands=1 << 23), norm(channels=4096, groups=1)), nb.EUNSUPPORTED, "8388607 workgroups")


def test_a_refused_read_leaves_the_streams_as_they_are():
    torch = pytest.importorskip("torch")
    held = layers.DecayState(2, 1, 8, device="cpu")
    held.state.fill_(7.0)
    held.pos.copy_(torch.tensor([-1, 0]))
    q = torch.zeros(1, 4, 1, 8)
    with pytest.raises(ValueError, match="cuda"):
        held.read(q, q, q, torch.tensor([0, 2, 4]), torch.zeros(1))
    assert held.pos.tolist() == [-1, 0] and (held.state == 7.0).all()
