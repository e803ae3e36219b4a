"""Where the sampling call's sums of masses would not fit in 64 bits it is refused, before any CUDA call (CPU only)."""
import ctypes

import pytest

from test_decode_checks import DUMMY, env, params  # noqa: F401


@pytest.mark.parametrize("how,refused", [
    (dict(top_p_all=0.9), True), (dict(top_p=DUMMY), True), (dict(top_p_all=0.9, temperature=DUMMY, temperature_all=0.0), True),
    (dict(top_p_all=0.9, top_k_all=50), True), (dict(), False), (dict(top_k_all=50, min_p_all=0.1), False),
    (dict(top_p_all=0.9, temperature_all=0.0), False)])
def test_vocabularies_with_a_top_p(env, how, refused):  # noqa: F811
    stride, decode, L = env
    assert "#define STRIDE_MAX_TOP_P_VOCAB (1 << 23) " in (stride._build.INCLUDE / "stride_decode.h").read_text()
    assert stride.MAX_TOP_P_VOCAB == 1 << 23
    p = ctypes.byref(params(decode, **how))
    call = lambda V: L.stride_sample(DUMMY, 0, V, V, 0, DUMMY, V, p, DUMMY, None, None, None)  # noqa: E731  (no rows: nothing is launched)
    assert call(1 << 23) == 0
    assert call((1 << 23) + 1) == call(1 << 30) == (stride.ERR_INVALID_ARG if refused else 0)
