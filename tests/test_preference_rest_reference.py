"""CPU: refusals of the preference loss's clear_rest."""
import ctypes

import __graft_entry__ as entry
from paper_2511_00874_b200 import binding

P = 1 << 20                      # an "aligned pointer": the calls below must return before it is used


def test_clear_rest_is_a_truth_value():
    entry.build()
    L = binding.lib()
    need = int(L.srq_preference_workspace_bytes(4))
    for clear in (2, -1):
        h = binding._Preference(1.0, 0.1, 0.0, clear)
        assert int(L.srq_preference_loss(P, 1, 4, 40, 40, P, 1, P, P, 1, 2, ctypes.byref(h), P, P, P, 2 * P, 40, P, need, None, None)) == binding.ERR_INVALID_ARG
