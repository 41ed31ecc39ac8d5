"""Native argument marshalling of the block operators: what it hands back to the general path, which then says what is wrong."""
import ctypes

import pytest
import torch


def test_the_step_takes_its_own_structures_only():
    import paper_1412_6249_amd as pa
    from paper_1412_6249_amd import _marshal
    desc, table = pa.adamw_desc(1e-3), pa.adamw_params([], [], [], []).array
    one = (pa.purine_adamw_param * 1)()
    conv = (pa.purine_conv_desc * 4)()
    assert _marshal.purine_adamw_step(desc, table, None, 0) == 0
    assert _marshal.purine_adamw_step(desc, one, None, 0) == pa.purine_adamw_step.__globals__["_lib"].purine_adamw_step(
        ctypes.byref(desc), one, 1, None, 0) != 0
    for bad in (None, b"", bytearray(ctypes.sizeof(one)), conv, one[0], [], ctypes.cast(one, ctypes.POINTER(pa.purine_adamw_param))):
        assert _marshal.purine_adamw_step(desc, bad, None, 0) is None
    for bad in (None, pa.conv_desc(), bytes(ctypes.sizeof(desc)), object()):
        assert _marshal.purine_adamw_step(bad, table, None, 0) is None
    assert _marshal.purine_adamw_step(desc, table, torch.zeros(1, dtype=torch.int32), 0) is None     # not on the device
    assert _marshal.purine_adamw_step(desc, table, None) is None and _marshal.purine_adamw_step(desc, table, None, 0, 0) is None
    with pytest.raises(TypeError):
        _marshal.adamw_types(1, 2)
    with pytest.raises((TypeError, ctypes.ArgumentError, AttributeError)):
        pa.purine_adamw_step(desc, None)


def test_operators_hand_back_what_is_not_on_the_device():
    from paper_1412_6249_amd import _marshal
    x = torch.zeros(4, 8)
    assert _marshal.purine_linear_fwd(x, x, None, None, x, None, 0, None, 0) is None
    assert _marshal.purine_linear_bwd_data(x, x, None, x, 0, 0.0, None, 0) is None
    assert _marshal.purine_linear_bwd_weight(x, x, x, None, 0.0, None, 0) is None
    assert _marshal.purine_act_bwd(x, x, x, None, 0, None, 0) is None
    assert _marshal.purine_group_norm_fwd(x, None, None, x, None, None, 2, 1e-5, 0, None, 0) is None
