"""Layers with weights of 4 bits: sizes and refusals (validation on the host, no GPU needed)."""
import ctypes

import pytest

P = [ctypes.c_void_p(0x10000000000 + (i << 40)) for i in range(8)]      # aligned, far apart, never dereferenced


@pytest.fixture(scope="module")
def ebs():
    import paper_2003_07577_b200 as pkg
    pkg.build()
    return pkg.binding


def off(p, n):
    return ctypes.c_void_p(p.value + n)


def ref(d):
    return None if d is None else ctypes.byref(d)


def pack(ebs, q, w=P[0], dtype=0, ldw=0, packed=P[1]):
    return ebs.lib().ebs_pack_weights_q4(w, dtype, ref(q), ldw, packed, None)


def unpack(ebs, q, w=P[0], dtype=0, ldw=0, packed=P[1]):
    return ebs.lib().ebs_unpack_weights_q4(packed, ref(q), w, dtype, ldw, None)


def forward(ebs, d, q, x=P[0], packed=P[1], bias=None, res=None, offsets=None, y=P[2], ws=P[7], ws_bytes=1 << 36):
    return ebs.lib().ebs_linear_q4_forward(x, packed, bias, res, offsets, ref(d), ref(q), y, ws, ws_bytes, None)


def test_sizes(ebs):
    q = ebs.q4_desc(4096, 4096, 128, ebs.EBS_BF16)
    codes, scales = 4096 * 4096 // 2, 4096 * 32 * 2
    assert ebs.ebs_q4_packed_bytes(q) == codes + scales
    q = ebs.q4_desc(17, 65, 32, ebs.EBS_F32, 3)                         # whole tiles of 16 x 64, groups of a row rounded up
    assert ebs.ebs_q4_packed_bytes(q) == 3 * 2 * 2 * 512 + (3 * 2 * 3 * 16 * 4 + 255) // 256 * 256
    assert ebs.ebs_linear_q4_workspace_bytes(ebs.linear_desc(5, 17, 65, ebs.EBS_F32), q) == (5 * 72 * 4 + 255) // 256 * 256
    assert ebs.ebs_linear_q4_workspace_bytes(ebs.linear_desc(1, 17, 65, ebs.EBS_F32), q) == 0          # one row starts where x does
    assert ebs.ebs_linear_q4_workspace_bytes(ebs.linear_desc(5, 17, 65, ebs.EBS_F32, ldx=68), q) == 0


@pytest.mark.parametrize("change", [dict(n=0), dict(k=0), dict(experts=0), dict(experts=-3), dict(group=16), dict(group=0), dict(group=256), dict(group=48), dict(dtype=1),
                                    dict(dtype=2), dict(dtype=5), dict(dtype=-1)])
def test_descriptors(ebs, change):
    bad = ebs.EBS_ERR_INVALID_ARG
    args = dict(n=64, k=128, group=64, dtype=ebs.EBS_F16, experts=1)
    q = ebs.q4_desc(**{**args, **change})
    d = ebs.linear_desc(4, q.n, q.k, q.dtype)
    assert pack(ebs, q) == unpack(ebs, q) == forward(ebs, d, q) == bad
    assert ebs.ebs_q4_packed_bytes(q) == ebs.ebs_linear_q4_workspace_bytes(d, q) == 0


def test_sizes_beyond_the_index_range(ebs):
    for args in (dict(n=(1 << 30) + 1, k=1, group=32), dict(n=1, k=(1 << 30) + 1, group=32), dict(n=1 << 20, k=1 << 20, group=32, experts=2), dict(n=1 << 29, k=1, group=32, experts=1 << 11)):
        q = ebs.q4_desc(**args)
        assert pack(ebs, q) == unpack(ebs, q) == ebs.EBS_ERR_OVERFLOW and ebs.ebs_q4_packed_bytes(q) == 0
    q = ebs.q4_desc(1 << 20, 64, 64)
    assert pack(ebs, q, ldw=1 << 21) == ebs.EBS_ERR_OVERFLOW
    q = ebs.q4_desc(1 << 20, 64, 64)
    assert forward(ebs, ebs.linear_desc(1 << 30, 1 << 20, 64, ebs.EBS_F32, ldy=1 << 20), q) == ebs.EBS_ERR_OVERFLOW      # y


def test_refusals(ebs):
    bad = ebs.EBS_ERR_INVALID_ARG
    q = ebs.q4_desc(64, 128, 64, ebs.EBS_F16)
    for call in (pack, unpack):
        for change in (dict(w=None), dict(packed=None), dict(dtype=1), dict(dtype=7), dict(ldw=127), dict(ldw=-1), dict(w=off(P[0], 2)), dict(packed=off(P[1], 8)), dict(packed=P[0]),
                       dict(w=off(P[1], 64 * 64))):
            assert call(ebs, q, **change) == bad, change
        assert call(ebs, None) == bad
    d = ebs.linear_desc(4, 64, 128, ebs.EBS_F16, ldx=129)
    need = ebs.ebs_linear_q4_workspace_bytes(d, q)
    assert need > 0
    for change in (dict(x=None), dict(packed=None), dict(y=None), dict(x=off(P[0], 2)), dict(packed=off(P[1], 4)), dict(y=off(P[2], 8)), dict(bias=off(P[3], 4)),
                   dict(res=off(P[3], 4)), dict(offsets=off(P[4], 2)), dict(ws=None), dict(ws_bytes=need - 1), dict(ws=off(P[7], 8)), dict(y=P[0]), dict(y=P[1]), dict(bias=P[2]),
                   dict(res=off(P[2], 16)), dict(ws=P[2]), dict(ws=P[0]), dict(ws=P[1]), dict(offsets=P[2]), dict(offsets=off(P[2], 4 * 64 * 2 - 4)), dict(offsets=P[7])):
        assert forward(ebs, d, q, **change) == bad, change
    assert forward(ebs, None, q) == bad and forward(ebs, d, None) == bad
    for other in (ebs.linear_desc(4, 65, 128, ebs.EBS_F16), ebs.linear_desc(4, 64, 127, ebs.EBS_F16), ebs.linear_desc(4, 64, 128, ebs.EBS_BF16),
                  ebs.linear_desc(-1, 64, 128, ebs.EBS_F16), ebs.linear_desc(4, 64, 128, ebs.EBS_F16, act=5), ebs.linear_desc(4, 64, 128, ebs.EBS_F16, ldy=63)):
        assert forward(ebs, other, q) == bad and ebs.ebs_linear_q4_workspace_bytes(other, q) == 0
    assert forward(ebs, d, ebs.q4_desc(64, 128, 64, ebs.EBS_F16, 2)) == bad                            # experts without offsets
    assert forward(ebs, ebs.linear_desc(0, 64, 128, ebs.EBS_F16), q, x=None, y=None, ws=None, ws_bytes=0) == ebs.EBS_OK       # no rows: nothing is launched


def test_fast_path_types(ebs):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(ebs.__file__), "_fastcall.so")
    spec = importlib.util.spec_from_file_location("_fastcall", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    for call, args in ((m.pack_weights_q4, (None, 0, None, 0, None, None)), (m.unpack_weights_q4, (None, None, None, 0, 0, None)),
                       (m.linear_q4_forward, (None,) * 10), (m.clip_gradients, (None, 0, 1.0, None, None, None))):
        with pytest.raises((RuntimeError, TypeError)):                  # not bound yet, or a descriptor of another type
            call(*args)
        with pytest.raises(TypeError):
            call(None)
