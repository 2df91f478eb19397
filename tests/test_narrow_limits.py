"""The largest calls of the entry points of 8 and 4 bits, on the host: those whose launch would
have 2^32 threads are refused, not handed to the device."""
import pytest

from test_narrow_host import CACHE, G, _err, caller, lib  # noqa: F401

MOST = 1 << 28
FAR = 1 << 44  # (behind all caches and indices, tensors of 2^39 bytes apart)


def _write(lib):
    return caller(lib, "kv_write_fp4", dict(k=FAR, v=2 * FAR, kvs=1024, **CACHE, slots=5 * G, T=64, Hkv=8, D=128, bs=16,
                                            nb=512, dt=1))


def _read(lib):
    return caller(lib, "kv_read_fp4", dict(**CACHE, tab=5 * G, cu=6 * G, first=7 * G, k=FAR, v=2 * FAR, kvs=1024, B=4, T=64,
                                           Hkv=8, D=128, bs=16, mb=64, nb=512, dt=1))


@pytest.mark.parametrize("name,make", [("kv_write_fp4", _write), ("kv_read_fp4", _read)])
def test_tokens_of_a_cache_call(lib, name, make):
    """Workgroups of 256 threads take 16 tokens of heads of 128: 2^28 - 15 tokens and more are 2^24 of them."""
    call = make(lib)
    for T in (MOST - 15, MOST - 1, MOST):
        assert call(T=T) == 1 and name in _err(lib) and "2^28" in _err(lib), (T, _err(lib))
    # the last that fit pass this check (what refuses them is the null address)
    for T, D in ((MOST - 16, 128), (MOST - 1, 64)):
        assert call(T=T, D=D, kc=None) == 1 and "null" in _err(lib), (T, D, _err(lib))
    assert call(T=MOST, D=64) == 1 and "2^28" in _err(lib)
