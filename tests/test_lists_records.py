"""Records of tensors (rocket_tensor) as the C ABI takes them; needs no GPU: a call that is refused has launched nothing."""
import ctypes

import numpy as np

from paper_2301_08527_amd import rocket

RECORD = np.dtype([("data", np.uint64), ("count", np.int64), ("dtype", np.int32), ("reserved", np.int32)])
P = ctypes.c_void_p(4096)


def test_the_reserved_field_is_0():
    """of every list, also of a tensor without values"""
    lib = rocket.load_library()
    good = np.array([(1 << 20, 100, 0, 0), (1 << 21, 0, 0, 0)], RECORD)
    for i in range(2):
        bad = good.copy()
        bad["reserved"][i] = 1
        assert lib.rocket_grad_workspace_bytes(bad.ctypes.data, 2) == 0
        for rc in (lib.rocket_grad_norm(bad.ctypes.data, 2, 1.0, P, P, 1 << 30, None),
                   lib.rocket_grad_clip(bad.ctypes.data, None, 2, 1.0, P, P, 1 << 30, None),
                   lib.rocket_grad_clip(good.ctypes.data, bad.ctypes.data, 2, 1.0, P, P, 1 << 30, None),
                   lib.rocket_sgd_tensors(bad.ctypes.data, good.ctypes.data, None, 2, 0.1, None, None),
                   lib.rocket_sgd_tensors(good.ctypes.data, bad.ctypes.data, None, 2, 0.1, None, None),
                   lib.rocket_sgd_tensors(good.ctypes.data, good.ctypes.data, bad.ctypes.data, 2, 0.1, None, None)):
            assert rc == rocket.ROCKET_EINVAL and "tensor %d: reserved" % i in rocket.rocket_last_error()
