"""What the operators around the path refuse, on the host: the C ABI's status codes before anything is
enqueued, and the binding's checks of tensors (CPU)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2609_36938_amd as janus
from plain import page_grow, positions, rotate

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced on the host
ODD = ctypes.c_void_p(0x1002)
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(janus.LIB_PATH):
        from paper_2609_36938_amd import build
        build.build()
    return janus.lib()


def _batch(total_q=4, max_ctx=100, B=1, es=0):
    b = janus._Batch(B, total_q, total_q, max_ctx, max_ctx, FAKE.value, FAKE.value, FAKE.value, FAKE.value, es)
    return b


def _rotary(dim=64, offset=0, layout=0, freq=FAKE.value):
    return janus._Rotary(dim, offset, layout, 0, 1.0, freq, None)


def test_page_grow(L):
    def call(b=_batch(), page=64, fl=FAKE, n=8, head=None, pt=FAKE, ld=2, slots=FAKE, counts=ctypes.c_void_p(0x2000)):
        return L.janus_page_grow(None if b is None else ctypes.byref(b), page, fl, n, head, pt, ld, slots, counts, None)

    assert call(b=None) == INVALID
    assert call(page=48) == INVALID and call(page=0) == INVALID
    assert call(fl=None) == INVALID and call(n=-1) == INVALID
    assert call(pt=None) == INVALID and call(slots=None) == INVALID and call(counts=None) == INVALID
    assert call(ld=1) == INVALID                                  # 64 ids for sessions of 100
    assert call(head=ctypes.c_void_p(0x2004)) == INVALID          # inside counts
    assert call(b=_batch(es=17)) == INVALID


def test_rope(L):
    def call(b=_batch(), r=_rotary(), x=FAKE, xdt=1, heads=2, size=64, out=ctypes.c_void_p(0x9000), odt=1, st=(128, 64),
             ost=(128, 64), scale=None):
        return L.janus_rope(None if b is None else ctypes.byref(b), None if r is None else ctypes.byref(r), x, xdt, *st,
                            heads, size, out, odt, *ost, scale, None)

    assert call(b=None) == INVALID and call(r=None) == INVALID
    assert call(x=None) == INVALID and call(out=None) == INVALID
    for r in (_rotary(63), _rotary(0), _rotary(66), _rotary(64, 2), _rotary(64, -2), _rotary(64, 0, 2), _rotary(freq=None)):
        assert call(r=r) == INVALID
    assert call(heads=0) == INVALID and call(size=0) == INVALID
    assert call(st=(-1, 64)) == INVALID and call(ost=(128, -64)) == INVALID
    assert call(odt=2) == INVALID and call(odt=1, scale=FAKE) == INVALID    # a scale goes with fp8, and only with it
    assert call(xdt=7) == INVALID and call(odt=7) == INVALID
    for ost in ((0, 64), (128, 0), (64, 64), (127, 64), (64, 200)):         # outputs on top of each other
        assert call(ost=ost) == INVALID, ost
    assert call(xdt=2) == UNSUPPORTED
    assert call(out=FAKE, odt=0) == INVALID and call(out=FAKE, ost=(192, 64)) == INVALID  # in place: same type and strides
    assert call(r=_rotary(2048), size=4096, ost=(8192, 4096)) == UNSUPPORTED
    assert call(heads=1 << 12, size=1 << 13, ost=(1 << 25, 1 << 13)) == UNSUPPORTED
    assert call(b=_batch(total_q=0, max_ctx=0)) == OK                       # nothing to do


def test_kv_append(L):
    def call(b=_batch(), r=_rotary(64, 512), x=FAKE, xdt=1, rot=FAKE, size=576, rows=FAKE, n=100, out=FAKE, odt=1, rb=1152,
             scale=None, rs=512):
        return L.janus_kv_append(None if b is None else ctypes.byref(b), None if r is None else ctypes.byref(r), x, xdt, rs,
                                 rot, 576, size, rows, n, out, odt, rb, scale, None)

    assert call(b=None) == INVALID and call(out=None) == INVALID
    assert call(x=None) == INVALID                                 # the latent part is missing
    assert call(r=None) == INVALID                                 # x_rot without a rotation
    assert call(r=_rotary(64, 520)) == INVALID
    assert call(size=0) == INVALID and call(n=-1) == INVALID and call(rs=-1) == INVALID
    assert call(rb=1150) == INVALID and call(rb=1153) == INVALID
    assert call(odt=2, rb=576) == INVALID                          # no room for the scale
    assert call(odt=1, scale=FAKE) == INVALID
    assert call(xdt=2) == UNSUPPORTED
    assert call(odt=2, rb=581) == UNSUPPORTED and call(odt=2, rb=592, out=ODD) == UNSUPPORTED
    b = _batch()
    b.ctx_start = None
    assert call(b=b, rows=None) == INVALID
    assert call(b=_batch(total_q=0, max_ctx=0)) == OK


def test_prefix_attn(L):
    big = ctypes.c_size_t(1 << 40)

    def call(b=_batch(), q=FAKE, H=16, dqk=576, dv=512, k=FAKE, v=FAKE, rs=(576, 576), pt=FAKE, ld=2, page=64, prefix=0,
             out=FAKE, odt=1, ws=None, size=big):
        return L.janus_prefix_attn(None if b is None else ctypes.byref(b), q, H, dqk, dv, k, v, *rs, pt, ld, page, prefix,
                                   ctypes.c_float(0.1), out, odt, None, ws, None if size is None else ctypes.byref(size),
                                   None)

    assert call() == OK                                            # a size query
    for name in ("b", "q", "k", "v", "pt", "out", "size"):
        assert call(**{name: None}) == INVALID, name
    assert call(H=0) == INVALID and call(page=3) == INVALID and call(ld=1) == INVALID
    assert call(rs=(500, 576)) == INVALID and call(rs=(576, 500)) == INVALID
    assert call(prefix=-1) == INVALID and call(prefix=101) == INVALID
    assert call(H=129) == UNSUPPORTED and call(odt=2) == UNSUPPORTED
    assert call(dqk=512) == UNSUPPORTED and call(dqk=128, dv=64) == UNSUPPORTED
    assert call(v=ctypes.c_void_p(0x2000)) == UNSUPPORTED          # MLA has one pool
    assert call(dqk=128, dv=128, v=ctypes.c_void_p(0x2000)) == OK
    assert call(rs=(580, 580)) == UNSUPPORTED
    for name in ("q", "k", "v", "out"):
        kw = {name: ODD}
        if name in "kv":
            kw = dict(k=ODD, v=ODD)
        assert call(**kw) == UNSUPPORTED, name
    assert call(b=_batch(total_q=1 << 28), H=16) == UNSUPPORTED    # rows beyond 32 bits
    long = _batch(total_q=1, max_ctx=100000)
    need = ctypes.c_size_t(0)
    assert call(b=long, ld=2000, size=need) == OK and need.value > 0 and need.value % (16 * 514 * 4) == 0
    short = ctypes.c_size_t(need.value - 1)
    assert call(b=long, ld=2000, size=short, ws=FAKE) == WORKSPACE
    assert call(b=long, ld=2000, ws=ctypes.c_void_p(0x1008), size=ctypes.c_size_t(need.value)) == UNSUPPORTED


def test_sizes_beyond_a_launch(L):
    """Refused before anything is enqueued: 2^24 tokens of rows, keys beyond 2^30."""
    many = _batch(total_q=1 << 24, max_ctx=1 << 24)
    r, big = _rotary(), ctypes.c_size_t(1 << 62)
    assert L.janus_rope(ctypes.byref(many), ctypes.byref(r), FAKE, 1, 64, 64, 1, 64, ctypes.c_void_p(0x9000), 1, 64, 64, None,
                        None) == UNSUPPORTED
    assert L.janus_kv_append(ctypes.byref(many), ctypes.byref(r), FAKE, 1, 64, None, 0, 64, FAKE, 100, FAKE, 1, 128, None,
                             None) == UNSUPPORTED
    far = _batch(total_q=1, max_ctx=(1 << 30) + 1)
    assert L.janus_prefix_attn(ctypes.byref(far), FAKE, 8, 128, 128, FAKE, FAKE, 128, 128, FAKE, 1 << 15, 1 << 16, 0,
                               ctypes.c_float(0.1), FAKE, 1, None, FAKE, ctypes.byref(big), None) == UNSUPPORTED


def test_frequencies(L):
    freq, mag = janus.rotary_frequencies(64, 10000.0)
    assert mag == 1.0 and np.allclose(freq, 10000.0 ** (-np.arange(32) / 32), rtol=1e-14)
    lin, mag = janus.rotary_frequencies(64, 10000.0, "linear", 8.0)
    assert mag == 1.0 and np.allclose(lin, freq / 8, rtol=1e-14)
    yarn, mag = janus.rotary_frequencies(64, 10000.0, "yarn", 40.0, 4096)
    assert abs(mag - (0.1 * math.log(40) + 1)) < 1e-6
    turns = 4096 * freq / (2 * math.pi)
    assert np.allclose(yarn[turns > 40], freq[turns > 40], rtol=1e-14)       # fast ones kept
    assert np.allclose(yarn[turns < 0.7], freq[turns < 0.7] / 40, rtol=1e-14)  # slow ones stretched
    assert (np.diff(yarn) < 0).all() and (yarn <= freq * (1 + 1e-14)).all() and (yarn >= freq / 40 * (1 - 1e-14)).all()
    for bad in (dict(dim=63), dict(dim=0), dict(base=1.0), dict(factor=0.5), dict(scaling="yarn"),
                dict(scaling="yarn", original_ctx=4096, beta_fast=1.0, beta_slow=1.0), dict(base=float("nan"))):
        with pytest.raises(janus.JanusError):
            janus.rotary_frequencies(**{**dict(dim=64), **bad})
    with pytest.raises(janus.JanusError):
        janus.rotary_frequencies(64, scaling="other")


def test_rotary_layout_matches_the_header(tmp_path):
    import os
    import subprocess
    src = tmp_path / "layout.c"
    names = [f[0] for f in janus._Rotary._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "janus.h"\nint main(void){\n'
                   + 'printf("%zu\\n", sizeof(janus_rotary));\n'
                   + "".join(f'printf("%zu\\n", offsetof(janus_rotary, {n}));\n' for n in names) + "return 0;}\n")
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.check_call(["gcc", "-std=c99", "-I", inc, "-o", str(tmp_path / "layout"), str(src)])
    got = [int(x) for x in subprocess.check_output([str(tmp_path / "layout")], text=True).split()]
    assert got[0] == ctypes.sizeof(janus._Rotary)
    assert got[1:] == [getattr(janus._Rotary, n).offset for n in names]


def test_binding_refuses_tensors_that_do_not_fit():
    """Wrong shapes, types and devices are refused before the library is called."""
    bt = janus.Batch([5], [3], device="cpu")
    rot = None
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(janus.JanusError):
        janus.Rotary(64, device="cpu")                              # frequencies belong on the GPU
    with pytest.raises(janus.JanusError):
        janus.Rotary(64, layout="other")
    for bad in (x[:2], x[0], x.half()):
        with pytest.raises(janus.JanusError):
            janus.rope(bt, rot, bad)
    with pytest.raises(janus.JanusError):
        janus.rope(bt, rot, x, out_dtype="int8")
    with pytest.raises(janus.JanusError):
        janus.rope(bt, rot, x, out=torch.zeros(3, 2, 32, dtype=torch.bfloat16))
    with pytest.raises(janus.JanusError):
        janus.rope(bt, rot, x, out_scale=torch.zeros(3))
    with pytest.raises(janus.JanusError):
        janus.kv_append(bt, None, x[:, 0])
    with pytest.raises(janus.JanusError):
        janus.kv_append(bt, x[:, 0], torch.zeros(10, 32, dtype=torch.bfloat16))
    with pytest.raises(janus.JanusError):
        janus.kv_append(bt, x[:, 0], torch.zeros(10, 64, dtype=torch.bfloat16), x_rot=x[:, 1])
    with pytest.raises(janus.JanusError):
        janus.kv_append(bt, x[:, 0], torch.zeros(7, 64, dtype=torch.bfloat16))  # 8 keys
    with pytest.raises(janus.JanusError):
        janus.kv_append(bt, x[:, 0], torch.zeros(10, 64, dtype=torch.bfloat16), rows=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(janus.JanusError):
        janus.kv_append(bt, x[:, 0, :0], torch.zeros(10, 0, dtype=torch.bfloat16))      # rows of nothing
    table = torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(janus.JanusError):
        janus.page_grow(bt, 4, torch.zeros(9, dtype=torch.int32), table)        # not on a GPU, and too narrow
    with pytest.raises(janus.JanusError):
        janus.prefix_attn(bt, x, x, x, table, 64, 0, 1.0, out_dtype="fp8")
    with pytest.raises(janus.JanusError):
        janus.prefix_attn(bt, x.float(), x, x, table, 64, 0, 1.0)


def test_the_plain_forms():
    """The tests' own forms on cases worked out by hand."""
    table = np.array([[4, -7, -7], [2, 3, -7]], np.int32)
    t, s, c = page_grow([2, 3], [1, 3], 2, 0, np.array([9, 8, 7], np.int32), 1, table)
    assert t.tolist() == [[4, 8, -7], [2, 3, 7]] and s.tolist() == [16, 7, 14, 15] and c.tolist() == [2, 3, 0]
    t, s, c = page_grow([2, 3], [1, 3], 2, 0, np.array([9, 8], np.int32), 1, table)
    assert t.tolist() == [[4, 8, -7], [2, 3, -7]] and s.tolist() == [16, 7, -1, -1] and c.tolist() == [1, 2, 1]
    assert positions([5, 0], [2, 1]).tolist() == [5, 6, 0]
    x = np.arange(1.0, 5.0)[None, None]
    y, _ = rotate(x, np.array([1]), np.array([math.pi / 2, math.pi]), 0, "half")
    assert np.allclose(y, [[[-3, -2, 1, -4]]])
    y, _ = rotate(x, np.array([1]), np.array([math.pi / 2, math.pi]), 0, "interleaved")
    assert np.allclose(y, [[[-2, 1, -3, -4]]])
    y, _ = rotate(x, np.array([1]), np.array([math.pi / 2]), 1, "half", 2.0, inverse=True)
    assert np.allclose(y, [[[1, 6, -4, 4]]])
