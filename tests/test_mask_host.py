"""The masks' definition against published answers of the generator, and what the dropout and feed-forward entry points refuse before
they touch a device."""
import ctypes as C
import os

import numpy as np
import pytest

import philox
from paper_2104_01981_amd import binding

F32, BF16, F16 = 0, 1, 2
EINVAL = binding.ECRM_EINVAL


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.library_path()):
        from paper_2104_01981_amd import build
        build.build()
    return binding.load_library()


@pytest.mark.parametrize("counter,key,answer", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_generator_of_the_masks(counter, key, answer):
    """The known answers of Philox 4x32-10 that its authors give."""
    assert tuple(int(x) for x in philox.philox(counter, key)) == answer


def test_masks_have_the_share_and_the_mean():
    for p in (0.1, 0.5, 0.9):
        k = philox.kept(p, 123, 456, 1000, 1000)
        # a million draws: five standard deviations
        assert abs(k.mean() - (1 - philox.border(p) / 65536)) < 5 * np.sqrt(p * (1 - p) / 1e6)
        assert abs((k * philox.factor(p)).mean() - 1) < 5 * np.sqrt(p / (1 - p) / 1e6)
    assert philox.kept(0.0, 1, 2, 3, 12).all() and not philox.kept(1.0, 1, 2, 3, 12).any()


def _mask(state=4096, offset=0, p=0.5):
    return binding.EcrmMask(state, offset, p)


@pytest.mark.parametrize("bad", [dict(mask=None), dict(mask=_mask(state=0)), dict(mask=_mask(state=4100)), dict(mask=_mask(p=-0.1)),
                                 dict(mask=_mask(p=1.5)), dict(mask=_mask(p=float("nan"))), dict(x=0), dict(x=8192 + 4), dict(x_stride=8),
                                 dict(x_stride=18), dict(x_stride=(1 << 48) + 4), dict(out=0), dict(out=65536 + 2), dict(out_stride=12),
                                 dict(type=3), dict(cols=0), dict(cols=6), dict(cols=(1 << 24) + 4), dict(rows=(1 << 32) + 1),
                                 dict(residual=131072 + 4, residual_stride=16), dict(residual=131072, residual_stride=8),
                                 dict(out=8192 + 8), dict(out=8192, out_stride=20), dict(residual=65536 + 16, residual_stride=16),
                                 dict(out=4096 - 64), dict(out=8192 + 16 * 2, x_stride=24, out_stride=28)])
def test_dropout_refuses(lib, bad):
    a = dict(mask=_mask(), x=8192, x_stride=16, residual=None, residual_stride=0, out=65536, out_stride=16, type=BF16, rows=5, cols=16)
    a.update(bad)
    assert lib.ecrm_dropout(a["mask"], a["x"], a["x_stride"], a["residual"], a["residual_stride"], a["out"], a["out_stride"], a["type"],
                            a["rows"], a["cols"], None) == EINVAL


def test_dropout_refuses_rows_that_no_memory_holds(lib):
    """As far apart as one row after another may be, but 2^20 of them: the last one's address passes 64 bits and comes round."""
    for rows, stride in ((1 << 20, 1 << 48), (1 << 32, 1 << 32), (3, (1 << 47) + 4)):
        assert lib.ecrm_dropout(_mask(), 8192, stride, None, 0, 65536, stride, F32, rows, 16, None) == EINVAL, (rows, stride)


def test_dropout_of_nothing(lib):
    assert lib.ecrm_dropout(_mask(), None, 0, None, 0, None, 0, F32, 0, 16, None) == 0


def test_lookup_with_dropout_refuses_without_a_context(lib):
    cfg = binding.EcrmConfig(rows=1 << 10, dim=36, k=4, servers=5, optimizer=0, lr=0.01, eps=1e-8, max_batch=64)
    ctx = C.c_void_p(0)
    assert lib.ecrm_create(C.byref(cfg), C.byref(ctx)) == 0
    m = _mask()
    for c, code in ((ctx, binding.ECRM_ENOTBOUND), (None, EINVAL)):
        assert lib.ecrm_embed_dropout(c, None, 1, 0, 1.0, 0, m, None, 0, 36, None) == code
        assert lib.ecrm_embed_grad_dropout(c, None, None, 0, 36, 1, 0, 1.0, m, None, None, None, None) == code
        assert lib.ecrm_embed_grad_dense_dropout(c, None, None, 0, 36, 1, 0, 1.0, m, None, 0, None) == code
    lib.ecrm_destroy(ctx)


def _create(lib, **kw):
    a = dict(dim=64, hidden=128, type=BF16, activation=0, max_rows=100, training=1)
    a.update(kw)
    out = C.c_void_p(0)
    return lib.ecrm_ffn_create(C.byref(binding.EcrmFfnConfig(**a)), C.byref(out)), out


@pytest.mark.parametrize("bad", [dict(dim=0), dict(dim=6), dict(dim=65540), dict(hidden=0), dict(hidden=10), dict(hidden=65540), dict(type=3),
                                 dict(activation=3), dict(max_rows=0), dict(max_rows=(1 << 26) + 1), dict(training=2)])
def test_feed_forward_refuses_its_configuration(lib, bad):
    rc, ffn = _create(lib, **bad)
    assert rc == EINVAL and not ffn.value


def test_feed_forward_on_the_host(lib):
    assert lib.ecrm_ffn_create(None, C.byref(C.c_void_p(0))) == EINVAL and lib.ecrm_ffn_bytes(None) == 0
    cfg = binding.EcrmFfnConfig(64, 128, BF16, 0, 100, 1)
    assert lib.ecrm_ffn_create(C.byref(cfg), None) == EINVAL
    rc, ffn = _create(lib)
    assert rc == 0
    # training takes room for three [100][128], one [100][64] more than h alone
    rc, small = _create(lib, training=0)
    assert rc == 0 and lib.ecrm_ffn_bytes(ffn) >= lib.ecrm_ffn_bytes(small) + 100 * (2 * 128 + 64) * 2
    assert lib.ecrm_ffn_bytes(small) >= 100 * 128 * 2
    size = lib.ecrm_ffn_bytes(ffn)
    w = dict(gate=1 << 30, gs=64, up=1 << 31, us=64, down=3 << 30, ds=128, work=1 << 32, size=size)

    def bind(**kw):
        a = {**w, **kw}
        return lib.ecrm_ffn_bind(ffn, a["gate"], a["gs"], a["up"], a["us"], a["down"], a["ds"], a["work"], a["size"])

    for bad in (dict(gate=0), dict(gate=(1 << 30) + 4), dict(gs=60), dict(gs=66), dict(gs=(1 << 20) + 4), dict(up=0), dict(us=32), dict(down=0),
                dict(ds=64), dict(gate=(1 << 32) + 256)):
        assert bind(**bad) == EINVAL, bad
    for bad in (dict(work=0), dict(work=(1 << 32) + 8), dict(size=size - 1)):
        assert bind(**bad) == binding.ECRM_ESCRATCH, bad
    for f, code in ((ffn, binding.ECRM_ENOTBOUND), (None, EINVAL)):
        assert lib.ecrm_ffn_forward(f, 4096, 64, 1, None, 0, None, 8192, 64, None, None) == code
        assert lib.ecrm_ffn_backward(f, 4096, 64, 8192, 16384, 64, 1, None, None, 0, 32768, 64, None, None, None, BF16, 0, None) == code
    assert lib.ecrm_ffn_bind(None, 0, 0, 0, 0, 0, 0, 0, 0) == EINVAL
    lib.ecrm_ffn_destroy(ffn)
    lib.ecrm_ffn_destroy(small)
    lib.ecrm_ffn_destroy(None)
