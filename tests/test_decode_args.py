"""Refusals of the operators around the decode step, and the rotary frequency tables: all of it on the host (CPU only)."""
import ctypes as C
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2605_29860_b200 as espo
from paper_2605_29860_b200 import build, decode

OK, NULL, DTYPE, SHAPE, ALIGN, CAPACITY, PARAM = 0, -1, -2, -3, -4, -5, -7
P = 1 << 20          # an address that is never read: every call below is refused, or has no rows


class Cache(C.Structure):
    _fields_ = espo.espo_kv_cache._fields_


class Rope(C.Structure):
    _fields_ = espo.espo_rope._fields_


class Seqs(C.Structure):
    _fields_ = espo.espo_sequences._fields_


@pytest.fixture(scope="module")
def lib():
    return C.CDLL(build.build())


def cache(**kw):
    d = dict(k=P, v=P, k_exp=None, v_exp=None, n_pages=10, page_size=64, n_kv_heads=2, head_dim=128, dtype=1, reserved=0)
    return Cache(**{**d, **kw})


def seqs(**kw):
    d = dict(pages=P, length=P, status=None, group=None, prefix_pages=None, prefix_length=None, max_pages=4, capacity=8,
             max_prefix_pages=0, n_groups=0)
    return Seqs(**{**d, **kw})


def i64(x):
    return C.c_int64(x)


def vp(x):
    return C.c_void_p(x)


def append(lib, c=None, rope=None, key=P, ks=256, value=P, vs=256, dtype=1, slots=P, pos=P, n=3, q=P, qs=512, hq=4, qo=P,
           qos=512, status=None):
    c = cache() if c is None else c
    return lib.espo_kv_append(C.byref(c) if c else None, C.byref(rope) if rope else None, vp(key), i64(ks), vp(value),
                              i64(vs), dtype, vp(slots), vp(pos), n, vp(q), i64(qs), hq, vp(qo), i64(qos), vp(status), None)


def append_rows(lib, c=None, s=None, n=3, rows=None, rope=None):
    c = cache() if c is None else c
    s = seqs() if s is None else s
    return lib.espo_kv_append_rows(C.byref(c), C.byref(rope) if rope else None, vp(P), i64(256), vp(P), i64(256), 1,
                                   C.byref(s) if s else None, vp(rows), n, None, i64(0), 0, None, i64(0), None, None)


@pytest.mark.parametrize("bad,code", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(dtype=0), DTYPE), (dict(dtype=3), DTYPE), (dict(dtype=2), NULL),
    (dict(dtype=2, k_exp=P), NULL), (dict(n_pages=0), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(page_size=48), SHAPE),
    (dict(page_size=8), SHAPE), (dict(head_dim=96), SHAPE), (dict(head_dim=256), SHAPE), (dict(k=P + 8), ALIGN),
    (dict(v=P + 2), ALIGN), (dict(dtype=2, k_exp=P + 1, v_exp=P), ALIGN), (dict(n_pages=1 << 30), CAPACITY),
    (dict(n_pages=2**31 - 1, n_kv_heads=2**31 - 1), CAPACITY), (dict(n_pages=(1 << 31) // 128), CAPACITY)])
def test_bad_caches_are_refused_everywhere(lib, bad, code):
    c = cache(**bad)
    assert append(lib, c) == code
    assert append_rows(lib, c) == code
    assert lib.espo_kv_gather(C.byref(c), vp(P), 3, vp(P), vp(P), 1, None, None) == code
    n = C.c_int64()
    assert lib.espo_attention_workspace(C.byref(c), 4, 4, C.byref(n)) == code


def test_append_refusals(lib):
    assert append(lib, n=0, key=None, value=None, q=None, qo=None, slots=None, pos=None) == OK
    for kw in (dict(key=None), dict(value=None), dict(q=None), dict(qo=None), dict(slots=None)):
        assert append(lib, **kw) == NULL, kw
    rope = Rope(P, 128, 0, 1.0, 0)
    assert append(lib, rope=rope, pos=None) == NULL
    assert append(lib, dtype=2) == DTYPE
    for kw in (dict(n=-1), dict(hq=-1), dict(ks=248), dict(vs=0), dict(qs=504), dict(qos=504), dict(ks=-256)):
        assert append(lib, **kw) == SHAPE, kw
    for kw in (dict(key=P + 8), dict(q=P + 4), dict(ks=260), dict(qos=516), dict(slots=P + 1), dict(pos=P + 2), dict(status=P + 1)):
        assert append(lib, **kw) == ALIGN, kw
    assert append(lib, hq=0, q=None, qo=None, qs=0, qos=0, n=0) == OK
    for r, code in ((Rope(None, 128, 0, 1.0, 0), NULL), (Rope(P, 0, 0, 1.0, 0), PARAM), (Rope(P, 12, 0, 1.0, 0), PARAM),
                    (Rope(P, 136, 0, 1.0, 0), PARAM), (Rope(P, 64, 0, math.nan, 0), PARAM), (Rope(P + 4, 64, 0, 1.0, 0), ALIGN)):
        assert append(lib, rope=r) == code


@pytest.mark.parametrize("bad,code", [
    (dict(length=None), NULL), (dict(pages=None), NULL), (dict(capacity=0), SHAPE), (dict(max_pages=-1), SHAPE),
    (dict(n_groups=-1), SHAPE), (dict(group=P, n_groups=2), NULL), (dict(group=P, n_groups=2, prefix_length=P, max_prefix_pages=1), NULL),
    (dict(max_pages=(1 << 23) + 1), CAPACITY), (dict(max_prefix_pages=(1 << 22) + 1), CAPACITY), (dict(length=P + 2), ALIGN),
    (dict(pages=P + 1), ALIGN)])
def test_bad_sequences_are_refused(lib, bad, code):
    s = seqs(**bad)
    assert append_rows(lib, s=s) == code
    assert attention(lib, s=s) == code


def test_append_rows_refusals(lib):
    assert append_rows(lib, n=9) == CAPACITY
    assert append_rows(lib, rows=P + 2) == ALIGN
    assert append_rows(lib, n=0) == OK
    assert lib.espo_kv_append_rows(C.byref(cache()), None, vp(P), i64(256), vp(P), i64(256), 1, None, None, 3, None, i64(0),
                                   0, None, i64(0), None, None) == NULL


def attention(lib, c=None, s=None, q=P, qs=512, hq=4, rows=None, n=3, scale=1.0, out=P, os=512, ws=P, wb=1 << 40, status=None):
    c, s = cache() if c is None else c, seqs() if s is None else s
    return lib.espo_attention(C.byref(c), C.byref(s), vp(q), i64(qs), hq, vp(rows), n, C.c_float(scale), vp(out), i64(os),
                              vp(ws), i64(wb), vp(status), None)


def test_attention_refusals(lib):
    assert attention(lib, n=0, q=None, out=None) == OK
    for kw in (dict(q=None), dict(out=None), dict(ws=None)):
        assert attention(lib, **kw) == NULL, kw
    for kw in (dict(hq=3), dict(hq=0), dict(hq=-2), dict(hq=130), dict(qs=504), dict(os=256), dict(n=-1)):
        assert attention(lib, **kw) == SHAPE, kw
    for kw in (dict(q=P + 8), dict(out=P + 2), dict(qs=516), dict(os=514), dict(ws=P + 128), dict(rows=P + 1), dict(status=P + 3)):
        assert attention(lib, **kw) == ALIGN, kw
    for scale in (math.nan, math.inf, -math.inf):
        assert attention(lib, scale=scale) == PARAM
    n = C.c_int64()
    assert lib.espo_attention_workspace(C.byref(cache()), 3, 4, C.byref(n)) == OK and n.value > 0
    assert attention(lib, wb=n.value - 1) == CAPACITY
    assert attention(lib, n=9) == CAPACITY
    assert lib.espo_attention_workspace(C.byref(cache()), 3, 4, None) == NULL
    assert lib.espo_attention_workspace(C.byref(cache()), -1, 4, C.byref(n)) == SHAPE


def sample(lib, x=P, dtype=1, stride=100, n=2, v=100, u=P, t=None, rows=None, status=None, cap=0, tok=P, logp=None, word=None, ws=P,
           wb=1 << 40):
    return lib.espo_sample(vp(x), dtype, i64(stride), n, v, vp(u), vp(t), None, None, None, vp(rows), vp(status), cap,
                           vp(tok), vp(logp), vp(ws), i64(wb), vp(word), None)


def test_sample_refusals(lib):
    assert sample(lib, n=0, x=None, u=None, tok=None, ws=None, wb=0) == OK
    for kw in (dict(x=None), dict(u=None), dict(tok=None), dict(ws=None)):
        assert sample(lib, **kw) == NULL, kw
    assert sample(lib, dtype=2) == DTYPE
    for kw in (dict(n=-1), dict(v=0), dict(stride=99), dict(status=P, cap=0)):
        assert sample(lib, **kw) == SHAPE, kw
    assert sample(lib, v=(1 << 19) + 1, stride=1 << 20) == CAPACITY
    for kw in (dict(x=P + 1), dict(dtype=0, x=P + 2), dict(u=P + 1), dict(t=P + 2), dict(tok=P + 3), dict(logp=P + 1), dict(word=P + 2), dict(ws=P + 64)):
        assert sample(lib, **kw) == ALIGN, kw
    n = C.c_int64()
    assert lib.espo_sample_workspace(2, 100, C.byref(n)) == OK and n.value > 0
    assert sample(lib, wb=n.value - 1) == CAPACITY
    assert lib.espo_sample_workspace(2, 100, None) == NULL
    assert lib.espo_sample_workspace(-1, 100, C.byref(n)) == SHAPE
    assert lib.espo_sample_workspace(1, 0, C.byref(n)) == SHAPE
    assert lib.espo_sample_workspace(1, (1 << 19) + 1, C.byref(n)) == CAPACITY


def test_gather_refusals(lib):
    g = lambda c=cache(), s=P, n=3, k=P, v=P, dt=1, w=None: lib.espo_kv_gather(C.byref(c), vp(s), n, vp(k), vp(v), dt, vp(w), None)  # noqa: E731
    assert g(n=0, s=None) == OK
    assert g(k=None, v=None) == OK
    assert g(s=None) == NULL
    assert g(dt=2) == DTYPE
    assert g(n=-1) == SHAPE
    assert g(k=P + 8) == ALIGN and g(v=P + 4) == ALIGN and g(s=P + 2) == ALIGN and g(w=P + 2) == ALIGN


def test_binding_refusals_without_a_device():
    import torch
    with pytest.raises(ValueError):
        espo.espo_kv_cache(torch.zeros(2, 2, 16, 64), torch.zeros(2, 2, 16, 64))
    with pytest.raises(ValueError):
        espo.espo_kv_cache(torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        espo.espo_sequences(torch.zeros(2, 3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        espo.espo_sample(torch.zeros(2, 3, dtype=torch.float16), torch.zeros(2), torch.zeros(2, dtype=torch.int32))


def test_frequencies():
    f, m = espo.espo_rope_frequencies(128, theta=1e6)
    i = np.arange(64)
    # pow() is good to a few units of 2^-53
    assert m == 1.0 and np.allclose(f.numpy(), 1e6 ** (-2.0 * i / 128), rtol=1e-14, atol=0)
    g, m = espo.espo_rope_frequencies(128, theta=1e6, kind=espo.ESPO_ROPE_LINEAR, factor=4.0)
    assert m == 1.0 and np.allclose(g.numpy(), f.numpy() / 4, rtol=1e-15, atol=0)
    # by parts: turns over the original context decide; fast pairs are kept, slow ones divided, a straight ramp between
    L, s = 4096.0, 8.0
    h, m = espo.espo_rope_frequencies(64, theta=1e4, kind=espo.ESPO_ROPE_BY_PARTS, factor=s, original_length=L)
    f, _ = espo.espo_rope_frequencies(64, theta=1e4)
    ratio = h.numpy() / f.numpy()
    turns = L * f.numpy() / (2 * math.pi)
    assert abs(m - (0.1 * math.log(s) + 1)) < 1e-6
    # the ramp's ends are rounded outwards to whole pairs, so a pair well past either border is decided by its turns alone
    assert np.allclose(ratio[turns > 64], 1.0, rtol=1e-14) and np.allclose(ratio[turns < 0.5], 1 / s, rtol=1e-14)
    assert np.all(np.diff(ratio) <= 1e-15)
    step = np.diff(ratio)[(ratio[:-1] < 1) & (ratio[1:] > 1 / s)]
    assert step.size > 2 and np.allclose(step, step[0], rtol=1e-9)
    one, _ = espo.espo_rope_frequencies(64, theta=1e4, kind=espo.ESPO_ROPE_BY_PARTS, factor=1.0)
    assert np.allclose(one.numpy(), f.numpy(), rtol=1e-14)


@pytest.mark.parametrize("kw", [dict(kind=3), dict(kind=-1), dict(theta=1.0), dict(theta=math.nan), dict(rot_dim=0), dict(rot_dim=12),
                                dict(rot_dim=-8), dict(kind=1, factor=0.5), dict(kind=1, factor=math.nan), dict(kind=2, factor=2.0, original_length=0.0),
                                dict(kind=2, factor=2.0, slow_turns=0.0), dict(kind=2, factor=2.0, fast_turns=1.0, slow_turns=1.0)])
def test_frequency_refusals(kw):
    with pytest.raises(espo.EspoError) as e:
        espo.espo_rope_frequencies(**{"rot_dim": 64, **kw})
    assert e.value.code == PARAM


def test_structures_of_another_device_are_refused(monkeypatch):
    """A cache or page table built on one device and used while another is current: refused before any address is passed on."""
    class Elsewhere:
        device = torch.device("cuda:1")

        def get_device(self):
            return 1

    def built(kind):
        x = kind.__new__(kind)
        x.tensors = (Elsewhere(),)
        return x

    monkeypatch.setattr(decode, "_current_device", lambda: 0)
    c, s, r = built(espo.espo_kv_cache), built(espo.espo_sequences), built(espo.espo_rope)
    z = torch.zeros(1, 1, 64)
    i = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: espo.espo_attention(c, s, z, z, z, 1.0), lambda: espo.espo_kv_gather(c, i, z),
                 lambda: espo.espo_kv_append(c, z, z, i), lambda: espo.espo_kv_append_rows(c, z, z, s),
                 lambda: espo.espo_kv_append(c, z, z, i, positions=i, rope=r)):
        with pytest.raises(ValueError, match="is on cuda:1, the current device is cuda:0"):
            call()


def test_attention_scales_that_leave_32_bits_are_refused(lib):
    """Scores are taken times log2(e) in 32 bits."""
    for scale in (2.0 ** 127, -2.0 ** 127, 2.0 ** -149, 0.0):
        assert attention(lib, n=0, q=None, out=None, scale=scale) == OK, scale
    for scale in (1.8e38, -1.8e38, 3.4e38):
        assert attention(lib, scale=scale) == PARAM, scale


def test_the_package_imports_where_torch_has_no_cuda():
    """A torch built without CUDA lacks its private device functions; the sharding helpers and generators work there."""
    code = """
import torch
for name in [n for n in dir(torch._C) if n.startswith("_cuda_")]:
    delattr(torch._C, name)
import paper_2605_29860_b200 as espo
from paper_2605_29860_b200 import shard, synth
try:
    espo.espo_kv_cache(*[torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16)] * 2)
except ValueError as e:
    print(e)
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(espo.__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True)
    assert r.returncode == 0 and "must be a CUDA tensor" in r.stdout, r.stderr
