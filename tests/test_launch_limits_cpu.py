"""Calls whose launch would have 2^32 threads and more are refused before any HIP
call: the runtime would run only some of them, without an error."""
from paper_2002_09049_amd import mpq


def _refused(rc):
    assert rc == mpq.MPQ_ERR_HIP and "invalid argument" in mpq.last_error(), (rc, mpq.last_error())


def test_reconstruct():
    lib = mpq.load()
    # one row of 4096 elements a workgroup of 256 threads
    _refused(lib.mpq_reconstruct(64, 64, 64, 1 << 24, 4096, 1, 64, None))


def test_integer_scales():
    lib = mpq.load()
    _refused(lib.mpq_integer_scales(64, 64, 1 << 28, 16, 8, 64, None, None))
