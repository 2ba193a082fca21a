"""MI355X-native MoE expert layer of one expert-parallel rank (ElasticMoE hot path).

`binding` mirrors the C ABI of libelasticmoe.so one to one; `layer.MoELayer` is a
small convenience holder of the device buffers (torch is used for memory and
streams only).  Beside the layer, as torch functions: `scaled` (8-bit operators), `dispatch` (tokens
sorted by expert and back, with gradients) and `four_bit` (experts held in 4 bits).
"""
from . import binding  # noqa: F401
from .binding import *  # noqa: F401,F403
