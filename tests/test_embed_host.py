"""Host side of the operators on embedding tables: sizes and null handles, without a device."""
import ctypes

import paper_2307_12059_amd as kgc


def test_sizes_of_workspaces_and_tables():
    assert kgc.kgc_lookup_grad_bytes(0, 10, 8) == 0 and kgc.kgc_lookup_grad_bytes(100, 10, 8) == 0          # few ids need none
    some = kgc.kgc_lookup_grad_bytes(100_000, 5000, 8)
    assert some >= 8 * 100_000 and some % 256 == 0
    assert kgc.kgc_lookup_grad_bytes(100_000, 1_000_000, 8) >= some
    for bad in ((-1, 1, 1), (1, -1, 1), (1, 1, 0), (1, 1, 961), (1 << 31, 1, 1)):
        assert kgc.kgc_lookup_grad_bytes(*bad) == 0
    assert kgc.kgc_table4_bytes(0, 8) == 0
    assert kgc.kgc_table4_bytes(1, 1) == 1152 and kgc.kgc_table4_bytes(64, 32) == 1152
    assert kgc.kgc_table4_bytes(65, 33) == 4 * 1152
    assert kgc.kgc_table4_bytes(-1, 8) == 0 and kgc.kgc_table4_bytes(8, 961) == 0


def test_null_handles_are_rejected_without_a_device():
    lib = kgc.load_library()
    assert lib.kgc_set_stream(None, None) == kgc.KGC_E_INVALID
    assert lib.kgc_lookup(None, None, 0, 0, None, 0, 1.0, None, 0, 0, None, 0, 1.0, 0, 1, None, 1, 0) == kgc.KGC_E_INVALID
    assert lib.kgc_lookup_grad(None, None, 0, 0, None, 0, 0, 1, 1.0, 0, None, 0, 0, 1, None, 0) == kgc.KGC_E_INVALID
    assert lib.kgc_pack4(None, None, 0, 0, 1, None, 0, None) == kgc.KGC_E_INVALID
    assert lib.kgc_scores4(None, None, 0, 1, None, 0, 0, 0, 1.0, None, 0.0, None, 0, 0) == kgc.KGC_E_INVALID
    assert lib.kgc_adjust(None, None) == kgc.KGC_E_INVALID
    assert lib.kgc_adjust(None, ctypes.byref(kgc.kgc_adjustment())) == kgc.KGC_E_INVALID
    assert ctypes.sizeof(kgc.kgc_adjustment) == 160
