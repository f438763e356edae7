"""What the serving step's entry points refuse before anything is enqueued (CPU)."""
import ctypes

import pytest
import torch

ca = pytest.importorskip("paper_2605_16839_amd")

FAKE = 0x1000    # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    return ca.load()


def _cache(**kw):
    base = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, max_kv_blocks=16, num_pages=99)
    base.update(kw)
    return ca.Cache(**base)


def _name(lib, status):
    return lib.ca_status_string(status).decode()


@pytest.mark.parametrize("kw,group,code", [
    (dict(), 0, "CA_OK"), (dict(), 2, "CA_OK"), (dict(num_q_heads=14), 7, "CA_OK"),
    (dict(head_dim=96), 0, "CA_ERR_UNSUPPORTED"), (dict(page_size=32), 0, "CA_ERR_UNSUPPORTED"),
    (dict(batch=0), 0, "CA_ERR_SHAPE"), (dict(num_kv_heads=3), 0, "CA_ERR_SHAPE"),
    (dict(max_kv_blocks=0), 0, "CA_ERR_SHAPE"), (dict(max_kv_blocks=16385), 0, "CA_ERR_SHAPE"),
    (dict(num_pages=0), 0, "CA_ERR_SHAPE"), (dict(v_layout=2), 0, "CA_ERR_SHAPE"),
    (dict(batch=1 << 30), 0, "CA_ERR_SHAPE"), (dict(num_q_heads=1 << 17), 0, "CA_ERR_SHAPE"), (dict(), 3, "CA_ERR_GROUP"), (dict(), 8, "CA_ERR_GROUP"),
])
def test_check_cache(lib, kw, group, code):
    assert _name(lib, lib.ca_check_cache(_cache(**kw).ref, group)) == code
    assert (lib.ca_last_error_detail().decode() == "") == (code == "CA_OK")


def _assign(lib, c, **kw):
    a = dict(new=FAKE, tokens=4, seq=FAKE, table=FAKE, free=FAKE, cap=8, count=FAKE, slots=FAKE,
             pos=FAKE, indptr=FAKE, granted=FAKE, seq_out=FAKE, count_out=FAKE)
    a.update(kw)
    return _name(lib, lib.ca_assign_slots(c, a["new"], a["tokens"], a["seq"], a["table"], a["free"],
                                          a["cap"], a["count"], a["slots"], a["pos"], a["indptr"],
                                          a["granted"], a["seq_out"], a["count_out"], None))


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), "CA_ERR_SHAPE"), (dict(cap=-1), "CA_ERR_SHAPE"),
    (dict(slots=FAKE + 4), "CA_ERR_UNALIGNED"),
] + [({k: None}, "CA_ERR_NULL") for k in ("new", "seq", "table", "free", "count", "slots", "pos",
                                         "indptr", "granted", "seq_out", "count_out")])
def test_assign_slots_refuses(lib, kw, code):
    assert _assign(lib, _cache().ref, **kw) == code


def test_null_cache(lib):
    assert _assign(lib, None) == "CA_ERR_NULL"
    assert _name(lib, lib.ca_check_cache(None, 0)) == "CA_ERR_NULL"
    assert lib.ca_decode_workspace_bytes(None, 0) == 0


@pytest.mark.parametrize("hole", range(7))
def test_release_pages_refuses(lib, hole):
    a = [FAKE] * 7
    a[hole] = None
    s = lib.ca_release_pages(_cache().ref, a[0], a[1], a[2], a[3], 8, a[4], a[5], a[6], None)
    assert _name(lib, s) == "CA_ERR_NULL"
    if hole == 0:
        s = lib.ca_release_pages(_cache().ref, *[FAKE] * 4, -1, *[FAKE] * 3, None)
        assert _name(lib, s) == "CA_ERR_SHAPE"


def _rotary(rot_dim=128, axes=1, pair_axis=None, inv_freq=FAKE):
    r = ca.Rotary(None, num_axes=axes)
    r.keep = (ctypes.c_int32 * 64)(*(pair_axis or []))
    if pair_axis is not None:
        r.c.pair_axis_host = ctypes.cast(r.keep, ctypes.POINTER(ctypes.c_int32))
    r.c.rot_dim, r.c.inv_freq = rot_dim, inv_freq
    return r


def _append(lib, r, T=3, q=FAKE, k=FAKE, v=FAKE, qs=1024, ks=256, vs=256, pos=FAKE, slots=FAKE,
            out=FAKE + 64, kp=FAKE, vp=FAKE):
    return _name(lib, lib.ca_rotary_append(_cache().ref, r, T, q, qs, k, ks, v, vs, pos, slots, out,
                                           kp, vp, None))


@pytest.mark.parametrize("kw,code", [
    (dict(rot_dim=130), "CA_ERR_UNSUPPORTED"), (dict(rot_dim=144), "CA_ERR_UNSUPPORTED"),
    (dict(rot_dim=24), "CA_ERR_UNSUPPORTED"), (dict(rot_dim=-16), "CA_ERR_UNSUPPORTED"),
    (dict(axes=0), "CA_ERR_UNSUPPORTED"), (dict(axes=5), "CA_ERR_UNSUPPORTED"),
    (dict(axes=2, pair_axis=[0, 2]), "CA_ERR_SHAPE"), (dict(axes=2, pair_axis=[0, -1]), "CA_ERR_SHAPE"),
    (dict(inv_freq=None), "CA_ERR_NULL"),
])
def test_rotary_refuses(lib, kw, code):
    assert _append(lib, _rotary(**kw).ref) == code


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), "CA_ERR_SHAPE"), (dict(T=(1 << 23) + 1), "CA_ERR_SHAPE"), (dict(qs=1016), "CA_ERR_SHAPE"), (dict(ks=248), "CA_ERR_SHAPE"),
    (dict(vs=0), "CA_ERR_SHAPE"), (dict(qs=1028), "CA_ERR_UNALIGNED"), (dict(ks=260), "CA_ERR_UNALIGNED"),
    (dict(q=FAKE + 8), "CA_ERR_UNALIGNED"), (dict(out=FAKE + 8), "CA_ERR_UNALIGNED"),
    (dict(vp=FAKE + 2), "CA_ERR_UNALIGNED"), (dict(slots=FAKE + 4), "CA_ERR_UNALIGNED"),
    (dict(out=FAKE, qs=2048), "CA_ERR_SHAPE"),     # q_out = q of a fused projection
] + [({n: None}, "CA_ERR_NULL") for n in ("q", "k", "v", "pos", "slots", "out", "kp", "vp")])
def test_rotary_append_refuses(lib, kw, code):
    assert _append(lib, _rotary().ref, **kw) == code


def test_rotary_append_of_nothing(lib):
    assert _append(lib, _rotary().ref, T=0, q=None, k=None, v=None, pos=None, slots=None, out=None) == "CA_OK"


def _decode(lib, q=FAKE, kp=FAKE, vp=FAKE, pt=FAKE, kl=FAKE, ip=None, ix=None, gs=0, scale=0.1, out=FAKE,
            ws=FAKE, nbytes=1 << 40):
    return _name(lib, lib.ca_decode_attention(_cache().ref, q, kp, vp, pt, kl, ip, ix, gs, scale, out,
                                              None, ws, nbytes, None))


@pytest.mark.parametrize("kw,code", [
    (dict(ip=FAKE), "CA_ERR_NULL"), (dict(ix=FAKE), "CA_ERR_NULL"), (dict(gs=-1), "CA_ERR_GROUP"),
    (dict(gs=3), "CA_ERR_GROUP"), (dict(scale=0.0), "CA_ERR_SHAPE"), (dict(scale=-1.0), "CA_ERR_SHAPE"),
    (dict(scale=float("nan")), "CA_ERR_SHAPE"), (dict(scale=float("inf")), "CA_ERR_SHAPE"),
    (dict(q=FAKE + 8), "CA_ERR_UNALIGNED"), (dict(out=FAKE + 2), "CA_ERR_UNALIGNED"),
    (dict(kp=FAKE + 8), "CA_ERR_UNALIGNED"), (dict(ws=FAKE + 8), "CA_ERR_WORKSPACE"),
    (dict(ws=None), "CA_ERR_WORKSPACE"), (dict(nbytes=1000), "CA_ERR_WORKSPACE"),
] + [({n: None}, "CA_ERR_NULL") for n in ("q", "kp", "vp", "pt", "kl", "out")])
def test_decode_attention_refuses(lib, kw, code):
    assert _decode(lib, **kw) == code


def test_decode_attention_refuses_rows_past_31_bits(lib):
    def status(batch, tables, group=0):
        c = _cache(batch=batch, max_kv_blocks=16384)
        t = FAKE if tables else None
        return _name(lib, lib.ca_decode_attention(c.ref, FAKE, FAKE, FAKE, FAKE, FAKE, t, t, group, 0.1,
                                                  FAKE, None, None, 0, None))
    assert status(1 << 17, False) == "CA_ERR_SHAPE"
    assert status((1 << 17) - 1, False) == "CA_ERR_WORKSPACE"       # the next check
    assert status(1 << 16, True) == "CA_ERR_SHAPE" and status(1 << 15, True, 2) == "CA_ERR_SHAPE"
    assert status((1 << 16) - 1, True) == "CA_ERR_WORKSPACE"


def test_binding_refuses_what_the_kernels_would_misread():
    c = _cache()
    cpu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="current device"):
        ca.release_pages(c, cpu, cpu, cpu, cpu, cpu)
    with pytest.raises(ValueError, match="float32"):
        ca.Rotary(torch.ones(32, dtype=torch.float64))
    with pytest.raises(ValueError, match="names 3 axes"):
        ca.Rotary(torch.ones(32), num_axes=3, pair_axis=[0, 1, 2])
    with pytest.raises(ca.CAError, match="must divide"):
        ca.check_cache(c, 3)
