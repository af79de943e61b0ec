"""Which tile the experts' products take: the query's refusals and the ends of its rules.  No GPU is needed."""
import pytest

from paper_1705_01598_amd import binding as B

TINY, SMALL, NARROW, WIDE = (64, 64), (128, 128), (128, 64), (256, 256)


def product(t, rows, experts, n):
    return B.tperm_expert_tile(False, B.TYPES[t], True, rows, experts, 100, n)


def gradient(t, experts, k, n):
    return B.tperm_expert_tile(True, B.TYPES[t], False, 1000, experts, k, n)


@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_tiles_of_16_bit_types(t):
    assert product(t, 0, 4, 64) == product(t, 1, 1, 1) == product(t, 63 * 64, 64, 4096) == TINY
    assert product(t, 64 * 64, 64, 4096) == product(t, 191 * 64, 64, 4096) == SMALL and product(t, 192 * 64, 64, 4096) == WIDE
    assert product(t, 1024 * 8, 8, 512) == SMALL and product(t, 1024 * 8, 8, 1024) == WIDE
    assert gradient(t, 8, 512, 512) == TINY and gradient(t, 16, 512, 512) == SMALL and gradient(t, 48, 512, 512) == WIDE


def test_tiles_of_32_bit_elements():
    assert product("f32", 63 * 64, 64, 4096) == TINY and product("f32", 64 * 64, 64, 4096) == NARROW
    assert gradient("f32", 7, 1024, 1024) == TINY and gradient("f32", 8, 1024, 1024) == NARROW


def test_the_query_refuses_what_the_calls_refuse():
    good = dict(gradient=False, dtype=B.TYPE_BF16, w_k_first=False, rows=8, experts=3, k=16, n=24)
    assert B.tperm_expert_tile(**good) == TINY
    for status, change in ((B.ERR_DIMS, dict(experts=0)), (B.ERR_DIMS, dict(experts=B.EXPERTS_MAX + 1)), (B.ERR_DIMS, dict(rows=-1)), (B.ERR_DIMS, dict(k=0)),
                           (B.ERR_DIMS, dict(n=B.WIDTH_MAX + 1)), (B.ERR_ELEM_SIZE, dict(dtype=3)), (B.ERR_TOO_LARGE, dict(rows=1 << 31))):
        with pytest.raises(B.TpermError) as e:
            B.tperm_expert_tile(**{**good, **change})
        assert e.value.status == status, change
