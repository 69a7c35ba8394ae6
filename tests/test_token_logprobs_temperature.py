"""The temperatures that mad_token_logprobs takes (no GPU: refused before anything is launched)."""
import ctypes

import pytest


@pytest.mark.parametrize("temperature", [2.0 ** -127, 5e-324, 2.0 ** 127, 1e300])
def test_temperatures_whose_factor_fp32_does_not_hold_are_refused(temperature):
    import paper_2608_30252_amd as mad
    p, temps = ctypes.c_void_p, (ctypes.c_double * 2)(1.0, temperature)
    lib = mad._load_library()
    assert lib.mad_token_logprobs(p(1 << 24), mad.MAD_F32, 1000, 1000, None, temps, 2, 1, 1000, 0, None, None, p(1 << 23), None, None,
                                  p(1 << 28), 1 << 30, None) == mad.MAD_EINVAL
    assert "temperature[1]" in lib.mad_last_error().decode()
