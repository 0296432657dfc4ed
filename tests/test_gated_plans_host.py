"""How the gated layers' products are dealt out, and how far their addresses reach: answers of the library without a GPU."""
import ctypes

import gated_forms
import pytest

from paper_1911_04477_amd import binding as B

LIMIT = (1 << 22) - 64  # the largest T, D and F


@pytest.mark.parametrize("T,D,F", [(1, 8, 64), (200, 64, 1000), (8192, 4096, 8192), (512, 1024, 2105377), (256, 2048, 2200001), (4096, 4096, 2200001),
                                   (512, 1024, LIMIT - 1), (8192, 4096, LIMIT)])
def test_offsets_of_a_tile_of_gradients(T, D, F):
    """A tile's last row of gradients begins (rows - 1) * 4 * F bytes after its first, F rounded up to 64, and its last piece 112 bytes
    further on; the reads take such an offset as 32 bits without a sign, and 16 bytes from there on stay below 2^32."""
    (form, _), _, largest = gated_forms.backward_plan(T, D, F)
    rows = min(T, (256, 128, 128, 64, 64)[form])
    assert largest == (rows - 1) * 4 * (-(-F // 64) * 64) + 112
    assert 0 <= largest <= 2 ** 32 - 1 - 16


def test_the_longest_rows_are_taken_by_the_largest_tiles():
    """The sizes above that pass 2^31 do so in 256-row tiles with a remainder of k."""
    for T, D, F in ((512, 1024, 2105377), (256, 2048, 2200001), (512, 1024, LIMIT - 1)):
        (form, _), _, largest = gated_forms.backward_plan(T, D, F)
        assert form == 0 and F % 64 and largest > 2 ** 31


def test_plans_of_refused_sizes():
    out = (ctypes.c_int64 * 5)()
    for sizes in ((0, 8, 8), (8, 0, 8), (8, 8, 0), (LIMIT + 1, 8, 8), (8, LIMIT + 1, 8), (8, 8, LIMIT + 1)):
        assert B.lib().bnn_testing_gated_backward_plan(*sizes, out) == -1
    assert B.lib().bnn_testing_gated_backward_plan(8, 8, 8, None) == -1


def test_workspaces_of_other_memory_are_refused():
    """Before anything else, so that no kernel gets an address of the host's memory."""
    import torch
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    saved, dh, ws = torch.zeros(2, 4, 4), torch.zeros(4, 4, dtype=torch.bfloat16), torch.zeros(1 << 16, dtype=torch.uint8)
    with pytest.raises(TypeError, match="workspace"):
        B.bnn_gated_ff_backward(x, x, x, saved, dh, workspace=ws)
    with pytest.raises(TypeError, match="workspace"):
        B.bnn_norm_gate_backward(x, x, x, x, workspace=ws)


def test_sizes_reach_every_form_of_the_forward_products():
    """What the GPU tests run: all nine with rows on 16 bytes, the four through registers."""
    for (weights, aligned), sizes in gated_forms.PRODUCTS.items():
        assert set(sizes) == (set(range(9)) if aligned else {1, 2, 4, 8})
        for form, (M, N) in sizes.items():
            assert gated_forms.product_form(M, N, weights, aligned) == form, (weights, aligned, form)


def test_sizes_reach_every_form_of_the_backward_products():
    """Each tile form, in one share of k and in several, with k in whole steps of 64 and with a remainder, and more steps than a ring has
    stages (four) in one share at least once each."""
    seen = {"dx": set(), "dw": set()}
    deep = {"dx": set(), "dw": set()}
    for T, D, F in gated_forms.BACKWARD:
        x, w, _ = gated_forms.backward_plan(T, D, F)
        for name, (form, shares), k, steps in (("dx", x, F, 2 * (F // 64)), ("dw", w, T, T // 64)):
            seen[name].add((form, shares > 1, k % 64 > 0))
            if steps // shares > 8:
                deep[name].add((form, k % 64 > 0))
    for name in seen:
        forms = {f for f, _, _ in seen[name]}
        assert forms == set(range(5)), (name, forms)
        assert {(f, cut) for f, _, cut in seen[name]} == {(f, cut) for f in range(5) for cut in (False, True)}, (name, seen[name])
        assert {(f, many) for f, many, _ in seen[name]} == {(f, many) for f in range(5) for many in (False, True)}, (name, seen[name])
        assert {f for f, _ in deep[name]} == set(range(5)), (name, deep[name])


def test_forms_of_refused_sizes():
    f = B.lib().bnn_testing_product_form
    assert f(0, 8, 1, 1, 256) == f(8, 0, 1, 1, 256) == f(8, 8, 3, 1, 256) == f(8, 8, 0, 1, 256) == f(8, 8, 1, 1, 0) == f(2 ** 31, 8, 1, 1, 256) == -1
