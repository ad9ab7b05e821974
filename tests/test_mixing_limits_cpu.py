"""The largest token mixing calls on the host: what a launch cannot hold is refused by the
workspace query and by the call alike, before anything is launched (the pointers
are never dereferenced)."""
import pytest

from test_mixing_cpu import UNSUPPORTED, backward, forward

# 2^21 sequences x value heads of 64 columns
MOST = dict(batch=1 << 17, k_heads=16, v_heads=16, v_size=64, tokens=17)


@pytest.mark.parametrize("kw,refused", [
    (dict(dtype=0, k_size=128), True),  # 16 columns a block: 2^23 blocks of 640 threads
    (dict(dtype=0, k_size=65), True), (dict(dtype=0, k_size=128, v_size=33), True),
    (dict(dtype=0, k_size=128, cu=1 << 20), True),
    (dict(dtype=0, k_size=128, v_size=32), False), (dict(dtype=0, k_size=64), False),
    (dict(dtype=1, k_size=128), False), (dict(dtype=2, k_size=128), False),
    (dict(dtype=0, k_size=128, tokens=16), False),  # token by token
    (dict(dtype=1, k_size=128, v_size=65), True)])
def test_forward(kw, refused):
    need = forward(query=True, **{**MOST, **kw})
    if refused:
        assert need == UNSUPPORTED and forward(**{**MOST, **kw}) == UNSUPPORTED
    else:
        assert need >= 0


@pytest.mark.parametrize("dtype", [0, 1])
def test_backward(dtype):
    assert backward(query=True, **MOST, dtype=dtype, k_size=128) > 0
    assert backward(query=True, **{**MOST, "v_size": 65}, dtype=dtype, k_size=128) == UNSUPPORTED
