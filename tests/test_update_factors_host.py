"""Update parameters that are each in range, but whose products an update would hold in fp32
as inf (and the weights as NaN), are refused on the host (no GPU needed; pointers are never read)."""
import ctypes

import paper_2505_17826_amd as R

FAKE = ctypes.c_void_p(0x1000)


def test_adamw():
    a = (R.rft_param * 1)(R.rft_param(0x1000, 0x2000, 0x3000, 0x4000, None, 10))
    for kw in (dict(lr=1e20, weight_decay=1e20), dict(lr=-1e20, weight_decay=1e20),
               dict(lr=1e25, beta1=1 - 1e-10, step=1)):
        h = R.adamw_params(**kw)
        assert R.lib().rft_adamw_step(a, 1, 0, 0, ctypes.byref(h), None, None) == R.RFT_E_PARAM, kw


def test_muon():
    m = R.rft_matrices(1, 8, 16, 16, 128)
    for kw in (dict(lr=1e20, weight_decay=1e20), dict(lr=1e20, scale=-1e20)):
        p = R.muon_params(**kw)
        assert R.lib().rft_muon_step(ctypes.byref(m), FAKE, 0, FAKE, FAKE, 0, None, ctypes.byref(p),
                                     None, None, 0, None) == R.RFT_E_PARAM, kw
