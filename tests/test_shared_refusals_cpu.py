"""What the operators around a shared cache refuse before they look for a GPU."""
import ctypes as C

import numpy as np
import pytest

import paper_2511_07423_amd as s
from paper_2511_07423_amd import binding as b


@pytest.mark.parametrize("bad", [
    dict(head_dim=0), dict(head_dim=63), dict(head_dim=64, rot_dim=66), dict(head_dim=64, rot_dim=31), dict(head_dim=64, rot_dim=0),
    dict(base=1.0), dict(base=0.0), dict(base=float("inf")), dict(base=float("nan")), dict(magnitude=float("nan")),
    dict(scaling=("linear", 0.0)), dict(scaling=("linear", -1.0)), dict(scaling=("linear", float("inf"))),
    dict(scaling=("bands", 8.0, 4.0, 4.0, 8192.0)), dict(scaling=("bands", 8.0, -1.0, 4.0, 8192.0)), dict(scaling=("bands", 8.0, 1.0, 4.0, 0.0)),
    dict(scaling=("bands", 0.0, 1.0, 4.0, 8192.0)), dict(inv_freq=np.full(32, np.nan))])
def test_rope_descriptions(bad):
    with pytest.raises(s.SyneraError) as e:
        s.Rope(**{**dict(head_dim=64), **bad})
    assert e.value.status == s.EINVAL


def test_rope_limits_and_words():
    with pytest.raises(s.SyneraError) as e:
        s.Rope(258)
    assert e.value.status == s.EUNSUP
    for bad in (dict(layout="other"), dict(scaling=("other", 1.0))):
        with pytest.raises(KeyError):
            s.Rope(64, **bad)
    for bad in (dict(scaling=("linear",)), dict(scaling=("bands", 1.0)), dict(inv_freq=np.ones(31))):
        with pytest.raises(ValueError):
            s.Rope(64, **bad)
    desc = b._RopeDesc(64, 64, 2, 0, 10000.0, 0, 0, 0, 0, 1.0, None)
    h = C.c_void_p(1)
    assert b._lib.synera_rope_create(C.byref(h), C.byref(desc)) == s.EINVAL and h.value is None
    desc.layout, desc.scaling = 0, 3
    assert b._lib.synera_rope_create(C.byref(h), C.byref(desc)) == s.EINVAL
    assert b._lib.synera_rope_create(C.byref(h), None) == s.EINVAL
    assert b._lib.synera_rope_create(None, C.byref(desc)) == s.EINVAL
    assert b._lib.synera_rope_destroy(None) == s.OK


@pytest.mark.parametrize("args,status", [((0, 1, 64, 1, 1, 1), s.EINVAL), ((4, 0, 64, 1, 1, 1), s.EINVAL), ((4, 4, 64, 0, 1, 1), s.EINVAL),
                                         ((4, 4, 64, 1, 0, 1), s.EINVAL), ((4, 4, 64, 1, 1, 0), s.EINVAL), ((4, 3, 64, 1, 1, 1), s.EUNSUP),
                                         ((4, 4, 96, 1, 1, 1), s.EUNSUP), ((2048, 8, 64, 1, 1, 1), s.EUNSUP),
                                         ((1024, 8, 64, 1, 1 << 20, 1), s.EUNSUP), ((4, 4, 64, 1 << 16, 1, 1 << 14), s.EUNSUP)])
def test_batch_limits(args, status):
    with pytest.raises(s.SyneraError) as e:
        s.SharedBatch(*args)
    assert e.value.status == status


def test_null_handles():
    lib, one = b._lib, b._pack_heads(16, 16, 0, 1, 64, 64, 64, 64)
    table, n = np.zeros((1, 1), np.int32), np.ones(1, np.int32)
    p = lambda a: a.ctypes.data_as(C.POINTER(C.c_int32))                                   # noqa: E731
    assert lib.synera_rope_apply(None, 0, 1, 16, one, None, None) == s.EINVAL
    assert lib.synera_qk_norm_rope(None, 0, 1, 16, one, None, 0.0, None) == s.EINVAL
    assert lib.synera_batch_plan(None, 1, p(n), p(n), p(table), 1, 1, None) == s.EINVAL
    assert lib.synera_append_rope(None, None, 0, one, one, one, 0.0, 16, 16, None) == s.EINVAL
    assert lib.synera_shared_attention(None, one, 16, 16, 0.0, None, None) == s.EINVAL
    assert lib.synera_batch_destroy(None) == s.OK
    assert lib.synera_batch_create(None, 4, 4, 64, 1, 1, 1) == s.EINVAL
    for args in ((1, None, p(n), p(table)), (1, p(n), None, p(table)), (1, p(n), p(n), None), (0, p(n), p(n), p(table))):
        assert lib.synera_validate_shared(*args, 1, 1, 1, 1) == s.EINVAL
    with pytest.raises(ValueError):
        s.validate_shared([1, 2], [1], table, 1, 1, 1)


def test_a_magnitude_has_to_be_finite_in_32_bits():
    for bad in (1e39, -1e300):
        with pytest.raises(s.SyneraError) as e:
            s.Rope(64, magnitude=bad)
        assert e.value.status == s.EINVAL
