"""Calls of the single layers that reach every kernel their plans pick.

test_layer_plans_cpu.py asks the library's plan headers which kernels calls can
reach and whether these reach them all; test_gpu_norm_forms.py and
test_gpu_adapter_forms.py run them.  A plan that picks further kernels needs
further calls here."""
import math

# Group norm: element type, channels, groups, and the elements of the vectors that
# the images' starts allow.  16-byte vectors whose channels share a group, or do
# not, or that take several pixels; the same in vectors of 8 and 4 bytes; single
# elements
NORM_CLASSES = [
    ("bf16", 64, 8, 8), ("f16", 64, 16, 8), ("bf16", 45, 5, 8), ("f16", 64, 8, 4),
    ("bf16", 45, 9, 4), ("bf16", 64, 16, 2), ("f16", 45, 5, 2), ("bf16", 64, 8, 1),
    ("f32", 32, 4, 4), ("f32", 32, 16, 4), ("f32", 45, 5, 4), ("f32", 32, 4, 2),
    ("f32", 45, 9, 2), ("f32", 32, 4, 1),
]


def norm_forms(backward):
    """(dtype, images, pixels, channels, groups, elements from one image's end to
    the next one's start): each class with up to 2 .. 20 vectors a thread
    (backward 10), then maps too large for registers, many and few.  The last
    step of pixels is ragged where vectors take several."""
    most_t, most_v = (512, 10) if backward else (1024, 20)
    forms = []
    for dtype, c, groups, ve in NORM_CLASSES:
        s = ve // math.gcd(ve, c)              # pixels of whole vectors
        lanes, most = 256 * ve // (s * c), most_t * ve // (s * c)  # of them at once
        sizes = [(256, v * lanes * s) for v in (2, 4, 6, 8)]
        sizes += [(512, v * most * s) for v in (10, 12, 16, 20) if v <= most_v]
        full = 4 if dtype == "f32" else 8
        sizes += [(512, (most_v + 3) * most * s), (2, 2 ** 16 * full // c)]
        for n, hw in sizes:
            pad = (ve % full - (hw - 1) * c) % full
            forms.append((dtype, n, hw - 1, c, groups, pad))
    return forms


# Adapters: rows, inputs, outputs, rank, adapters, type, elements between rows.
# Tiles of 256 outputs and 128 rows first (backward: inputs), whole and off every
# alignment; then smaller and split products and reductions.
ADAPTER_FORMS = [
    (2050, 1040, 3976, 12, 5, "bf16", 8), (2050, 1040, 3976, 12, 5, "f16", 1),
    (2050, 520, 3976, 16, 3, "f32", 4), (2050, 520, 3976, 5, 3, "f32", 1),
    (2050, 3976, 1040, 16, 70, "bf16", 0), (2050, 3976, 1040, 9, 5, "f16", 3),
    (2050, 3976, 520, 8, 40, "f32", 0), (2050, 3976, 520, 8, 5, "f32", 3),
    (262, 2056, 2064, 12, 1, "bf16", 0), (40, 2056, 32776, 8, 3, "bf16", 0),
    (132, 378, 234, 20, 2, "f32", 3), (81, 735, 556, 1, 1, "bf16", 3),
    (1, 1208, 1148, 4, 3, "f32", 4), (259, 504, 352, 5, 2, "f32", 0), (1, 1, 1, 4, 3, "bf16", 3),
    (1, 1, 1, 1, 4, "f32", 1), (1, 1024, 8, 5, 3, "bf16", 8), (468, 511, 1, 1, 3, "bf16", 1),
    (1, 4, 4, 8, 10, "f32", 0), (1, 8, 456, 8, 29, "bf16", 0), (1, 254, 268, 4, 5, "f32", 5),
    (257, 585, 1, 20, 5, "f32", 1), (1, 526, 556, 20, 29, "f16", 5), (17, 1, 1, 1, 1, "f32", 5),
    (19, 1, 1, 8, 2, "bf16", 3), (17, 4, 4, 8, 4, "f32", 0), (17, 8, 8, 5, 29, "f16", 0),
    (17, 256, 4, 5, 1, "f32", 4), (18, 456, 8, 12, 36, "bf16", 8),
    (135, 1025, 5581, 20, 9, "f32", 5),
]
