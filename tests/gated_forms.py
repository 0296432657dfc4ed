"""Sizes that reach every form of the 8-bit and gated layers' products, by the library's own rules (bnn_testing_product_form,
bnn_testing_gated_backward_plan) on a device of 256 compute units."""
import ctypes

from paper_1911_04477_amd import binding as B

UNITS = 256

# weights, rows on 16 bytes -> {form: (M, N)}
PRODUCTS = {
    (1, True): {0: (1030, 8200), 1: (1000, 4100), 2: (300, 16400), 3: (200, 4100), 4: (129, 3001), 5: (65, 3001), 6: (33, 520), 7: (700, 3001),
                8: (9, 1030)},
    (1, False): {1: (1000, 4100), 2: (700, 3001), 4: (300, 520), 8: (9, 1030)},
    (2, True): {0: (513, 8200), 1: (700, 3001), 2: (300, 8200), 3: (129, 3001), 4: (129, 1500), 5: (65, 1500), 6: (33, 520), 7: (200, 4100),
                8: (9, 1030)},
    (2, False): {1: (700, 3001), 2: (200, 4100), 4: (200, 1000), 8: (9, 1030)},
}

# T, D, F of backward passes
BACKWARD = [(4100, 2056, 1000), (4096, 2056, 1024), (1500, 2056, 8200), (700, 4104, 1000), (704, 4104, 1024), (4100, 200, 8200), (4096, 200, 8192),
            (8200, 2056, 1000), (2050, 72, 4099), (2048, 72, 4096), (500, 1032, 1000), (512, 1032, 1024), (1000, 2056, 2321), (200, 1032, 4099),
            (500, 200, 4099), (4100, 72, 520), (1500, 64, 72), (200, 64, 200), (192, 64, 512), (1000, 1024, 2321), (20, 2056, 200), (20, 2056, 2100),
            (256, 264, 4096), (130, 4104, 4099), (128, 1032, 4096), (4096, 264, 512), (4100, 64, 8200), (8192, 1032, 128)]


def product_form(M, N, weights, aligned, units=UNITS):
    return B.lib().bnn_testing_product_form(M, N, weights, int(aligned), units)


def backward_plan(T, D, F):
    """(form, shares) of the product that gives dx and of those that give the weights' gradients; the largest offset."""
    out = (ctypes.c_int64 * 5)()
    assert B.lib().bnn_testing_gated_backward_plan(T, D, F, out) == 0
    return (out[0], out[1]), (out[2], out[3]), out[4]
