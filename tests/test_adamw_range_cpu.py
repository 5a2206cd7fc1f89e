"""AdamW settings that leave fp32's range are refused (no GPU: every call fails
validation)."""
import ctypes

import pytest

import paper_2508_06993_amd as octnca
from paper_2508_06993_amd import _AdamW, _ParamList

GOOD = dict(lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, max_norm=1.0, scale=1.0,
            ema_decay=0.9)


@pytest.mark.parametrize("bad", [dict(lr=1e39), dict(weight_decay=1e39), dict(scale=1e39),
                                 dict(scale=1e-60), dict(eps=1e39), dict(lr=-1e-60)])
def test_settings_past_fp32(library_path, bad):
    plist = ctypes.byref(_ParamList(0x7f0000001000, 1, 10, 160, 2))      # never dereferenced
    assert octnca.lib().octree_nca_adamw(plist, ctypes.byref(_AdamW(**{**GOOD, **bad})),
                                         0x7f1000000000, None, None) == -1
