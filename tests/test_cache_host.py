"""CPU checks of the key/value cache: the oracle's own pins, the struct's layout and what
the library refuses before anything is queued."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import cache as oc


@pytest.fixture(scope="module")
def lib():
    from paper_2505_12398_gb300.build import build
    build()
    import paper_2505_12398_gb300 as tv
    return tv.library()


def test_format_pins():
    assert oc.e4m3_value(0x7e) == 448 and oc.e4m3_value(1) == 2.0 ** -9
    assert np.array_equal(oc.e4m3_byte(np.array([448.0, 1.0, 0.0])), [0x7e, 0x38, 0])
    x = np.array([6.0, -3, 2, 1.5, 0.25, 0.75, -1.25, 1.75, 2.5, 3.5, 5, 0, 0.26, 0.24, 4, -6])
    code, s = oc.quantize(x, 0)
    assert s == 1.0
    assert code.tolist() == [7, 13, 4, 3, 0, 2, 10, 4, 4, 6, 6, 0, 1, 0, 6, 15]
    assert np.array_equal(oc.held(x * 8, 3), oc.held(x, 0) * 8)
    assert np.array_equal(oc.held(x, 3), oc.held(x, 0))      # (its scale is 2^-3)


def test_bytes_round_trip():
    rng = np.random.default_rng(0)
    for d, P in ((64, 16), (128, 32)):
        block = np.zeros(P * d * 9 // 16, dtype=np.uint8)
        x = rng.standard_normal((P, d)) * np.exp2(rng.integers(-12, 12, (P, 1)))
        for slot in range(P):
            oc.put_row(block, P, slot, x[slot], -1)
        for slot in range(P):
            assert np.array_equal(oc.get_row(block, P, slot, d, -1), oc.held(x[slot], -1))


def test_half_step_of_the_format():
    """A held value is within half a step of e2m1 and of the scale's rounding: of the group's
    largest magnitude at most 1 / 6 + 2^-4."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((200, 64))
    err = np.abs(oc.held(x, 0) - x).reshape(200, 4, 16)
    top = np.abs(x).reshape(200, 4, 16).max(axis=-1, keepdims=True)
    assert np.all(err <= (1 / 6 + 2.0 ** -4) * top)


def test_masks_of_trees_and_prompts():
    m = oc.visible([-1, 0, 0, 1], 2, 4)
    assert m.astype(int).tolist() == [[1, 1, 1, 0, 0, 0], [1, 1, 1, 1, 0, 0],
                                      [1, 1, 1, 0, 1, 0], [1, 1, 1, 1, 0, 1]]
    assert oc.visible(None, 0, 2).astype(int).tolist() == [[1, 0], [1, 1]]
    q = np.ones((1, 2, 4))
    v = np.arange(8.0).reshape(2, 1, 4)
    out = oc.attention(q, np.zeros((2, 1, 4)), v, np.ones((1, 2), bool), 1.0)
    assert np.allclose(out[0, 1], v.mean(axis=0)[0])
    assert np.all(oc.attention(q, v, v, np.zeros((1, 2), bool), 1.0) == 0)


def test_struct_layout():
    from paper_2505_12398_gb300._binding import _Cache
    assert ctypes.sizeof(_Cache) == 40 and _Cache.data.offset == 24


def test_the_library_refuses_without_a_handle(lib):
    """No handle, no arrays: an error code, and nothing runs."""
    from paper_2505_12398_gb300._binding import _Cache
    c = _Cache(1, 1, 1, 64, 16, 4096, 0)
    ref = ctypes.cast(ctypes.pointer(c), ctypes.c_void_p)
    z = None
    assert lib.tv_cache_write(z, ref, 0, 1, 1, 0, z, z, z, z, 1, z, z) == -1
    assert lib.tv_cache_read(z, ref, 0, 1, 1, 0, z, z, 1, z, z, z, z) == -1
    assert lib.tv_cache_accept(z, ref, 1, 1, z, z, 1, z, z, z, z) == -1


def test_the_binding_refuses():
    from paper_2505_12398_gb300 import KVCache

    class Fake:
        device = torch.device("cpu")

        def _float_code(self, t, name):
            if t.dtype not in (torch.bfloat16, torch.float32):
                raise ValueError(name)
            return 0

    for bad in (dict(head_dim=96), dict(page_size=24), dict(layers=0), dict(kv_heads=0)):
        args = dict(layers=1, pages=2, kv_heads=1, head_dim=64, page_size=16)
        args.update(bad)
        with pytest.raises(ValueError):
            KVCache(Fake(), **args)
    with pytest.raises(ValueError):
        KVCache(Fake(), 1, 2, 1, 64, page_size=16, data=torch.zeros(3, dtype=torch.uint8))
    c = KVCache(Fake(), 1, 2, 1, 64, page_size=16)
    k = torch.zeros(2, 3, 1, 64)
    n, table = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32)
    for call in (lambda: c.write(0, k, k.bfloat16(), n, table),
                 lambda: c.write(0, k.half(), k.half(), n, table),
                 lambda: c.write(0, k[:, ::2], k[:, ::2], n, table),
                 lambda: c.write(0, k, k, n.long(), table),
                 lambda: c.write(0, k, k, n[:1], table),
                 lambda: c.write(0, k, k, n, table[0]),
                 lambda: c.write(0, k, k, n, table, rows=n[:1]),
                 lambda: c.read(0, n, table, 4, dtype="fp16"),
                 lambda: c.read(0, n, table, 4, first=n.long()),
                 lambda: c.accept(n, n, n, table),
                 lambda: c.accept(table.long(), n, n, table)):
        with pytest.raises((ValueError, IndexError)):
            call()
