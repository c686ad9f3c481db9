"""What the token and gradient-list entry points refuse before they touch a device."""
import ctypes as C
import os

import pytest

from paper_2104_01981_amd import binding


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.library_path()):
        from paper_2104_01981_amd import build
        build.build()
    return binding.load_library()


def test_an_unbound_context_refuses(lib):
    cfg = binding.EcrmConfig(rows=1 << 10, dim=36, k=4, servers=5, optimizer=0, lr=0.01, eps=1e-8, max_batch=64)
    ctx = C.c_void_p(0)
    assert lib.ecrm_create(C.byref(cfg), C.byref(ctx)) == 0
    assert lib.ecrm_embed(ctx, None, 1, 0, 1.0, 0, None, 0, 36, None) == binding.ECRM_ENOTBOUND
    assert lib.ecrm_embed_grad(ctx, None, None, 0, 36, 1, 0, 1.0, None, None, None, None) == binding.ECRM_ENOTBOUND
    assert lib.ecrm_embed_grad_dense(ctx, None, None, 0, 36, 1, 0, 1.0, None, 0, None) == binding.ECRM_ENOTBOUND
    for call in (lambda: lib.ecrm_embed(None, None, 1, 0, 1.0, 0, None, 0, 36, None),
                 lambda: lib.ecrm_embed_grad(None, None, None, 0, 36, 1, 0, 1.0, None, None, None, None),
                 lambda: lib.ecrm_embed_grad_dense(None, None, None, 0, 36, 1, 0, 1.0, None, 0, None)):
        assert call() == binding.ECRM_EINVAL
    lib.ecrm_destroy(ctx)


def _create(lib, *tensors):
    table = (binding.EcrmTensor * max(1, len(tensors)))(*[binding.EcrmTensor(*t) for t in tensors])
    out = C.c_void_p(0)
    return lib.ecrm_grads_create(table, len(tensors), C.byref(out)), out


@pytest.mark.parametrize("bad", [(0, 5, 0, 0, 0), (4096, 5, 0, 0, 3), (4098, 5, 0, 0, 0), (4097, 5, 0, 0, 1),
                                 (4096, (1 << 48) + 1, 0, 0, 0), (4096, 10, 4, 5, 0), (4096, 10, 8, 0, 0), (4096, 10, 8, 3, 0)])
def test_bad_tensors(lib, bad):
    rc, grads = _create(lib, (4096, 7, 0, 0, 0), bad)
    assert rc == binding.ECRM_EINVAL and not grads.value


def test_gradient_lists_on_the_host(lib):
    assert lib.ecrm_grads_create(None, 1, C.byref(C.c_void_p(0))) == binding.ECRM_EINVAL
    assert lib.ecrm_grads_create(None, 0, None) == binding.ECRM_EINVAL
    rc, grads = _create(lib, (4096, 1 << 30, 0, 0, 0), (0, 0, 0, 0, 1), (4098, 3, 0, 0, 2), (4096, 12, 8, 4, 1))
    assert rc == 0
    # a few words for each 16 KiB of a tensor, the list itself, and some room for sums
    assert (1 << 30) // 4096 * 4 < lib.ecrm_grads_bytes(grads) < (1 << 30) // 4096 * 64
    assert lib.ecrm_grads_norm(grads, 4096, None) == binding.ECRM_ENOTBOUND
    assert lib.ecrm_grads_clip(grads, None, 4096, 1.0, None) == binding.ECRM_ENOTBOUND
    assert lib.ecrm_grads_bind(grads, None, 1 << 30, None) == binding.ECRM_ESCRATCH
    assert lib.ecrm_grads_bind(grads, 4097, 1 << 30, None) == binding.ECRM_ESCRATCH
    assert lib.ecrm_grads_bind(grads, 4096, lib.ecrm_grads_bytes(grads) - 1, None) == binding.ECRM_ESCRATCH
    lib.ecrm_grads_destroy(grads)
    lib.ecrm_grads_destroy(None)
    assert lib.ecrm_grads_bytes(None) == 0
    assert lib.ecrm_grads_norm(None, 4096, None) == binding.ECRM_EINVAL
    assert lib.ecrm_grads_clip(None, None, 4096, 1.0, None) == binding.ECRM_EINVAL
    assert lib.ecrm_grads_bind(None, 4096, 0, None) == binding.ECRM_EINVAL


@pytest.mark.parametrize("dim,max_batch,updates,more", [(1024, 8192, 984064, True), (512, 8192, 876032, True), (256, 65536, 2916608, True),
                                                        (128, 100, 12032, False), (4, 1, 7168, False), (1024, 1 << 20, 114678784, True),
                                                        (128, 1 << 24, 531264512, False)])
def test_scratch_without_room_for_gradients(lib, dim, max_batch, updates, more):
    """Callers without gradient calls need what they needed before there were any; some geometries need no more with them."""
    cfg = binding.EcrmConfig(rows=1 << 22, dim=dim, k=4, servers=5, optimizer=0, lr=0.01, eps=1e-8, max_batch=max_batch)
    ctx = C.c_void_p(0)
    assert lib.ecrm_create(C.byref(cfg), C.byref(ctx)) == 0
    assert lib.ecrm_update_scratch_bytes(ctx) == updates
    every = lib.ecrm_scratch_bytes(ctx)
    assert every > updates if more else every == updates
    lib.ecrm_destroy(ctx)
    assert lib.ecrm_update_scratch_bytes(None) == 0 and lib.ecrm_scratch_bytes(None) == 0
