"""The C calls of the layers' operators by name, for tests: ``call(name, *arguments)`` raises ``TicTacError`` for a status."""

import ctypes

from paper_1803_03288_amd import binding

_I32, _I64, _PTR, _SIZE = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t

SIGNATURES = {
    "tictac_quantize_rows": (_I32, _I64, _I64, _PTR, _I64, _I32, _PTR, _I64, _PTR, _PTR),
    "tictac_dequantize_rows": (_I32, _I64, _I64, _PTR, _I64, _PTR, _I32, _PTR, _I64, _PTR),
    "tictac_layer_norm": (_I32, _I64, _I64, _PTR, _I64, _I32, _PTR, _PTR, ctypes.c_float, _PTR, _I64, _PTR, _PTR, _PTR, _I64, _PTR,
                          _PTR, _I64, _PTR, _PTR),
    "tictac_layer_norm_backward_workspace": (_I64, _I64, _PTR),
    "tictac_layer_norm_backward": (_I32, _I64, _I64, _PTR, _I64, _PTR, _I64, _PTR, _I64, _PTR, _I32, _PTR, _PTR, _PTR, _PTR, _I64,
                                   _PTR, _PTR, _PTR, _SIZE, _PTR),
    "tictac_linear_q8_workspace": (_I32, _I64, _I64, _I64, _PTR),
    "tictac_linear_q8": (_I32, _I64, _I64, _I64, _PTR, _I64, _PTR, _I64, _PTR, _PTR, _I64, _PTR, _I32, _PTR, _PTR, _I64, _PTR, _SIZE,
                         _PTR),
    "tictac_linear_q8_backward_workspace": (_I32, _I64, _I64, _I64, _PTR),
    "tictac_linear_q8_backward": (_I32, _I64, _I64, _I64, _PTR, _I64, _PTR, _I64, _PTR, _PTR, _I64, _PTR, _PTR, _I64, _PTR, _I64, _PTR,
                                  _PTR, _SIZE, _PTR),
}


def call(name, *args):
    fn = ctypes.CFUNCTYPE(_I32, *SIGNATURES[name])((name, binding.lib()))
    rc = fn(*args)
    if rc:
        binding._check(rc)
