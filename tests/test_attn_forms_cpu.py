"""Which form of the attention layer's kernels the GPU tests' cases take: the library's own rules (host code, no GPU)."""
import pytest

import test_gpu_attn_edges as edges
import test_gpu_attn_forms as forms
from routes import append_form, attn_plan


def paged_plan(c, dtype):
    B, S, Hq, Hk, Dh, page, window, lens, _ = c
    return attn_plan(B, S, Hq, Hk, Dh, (-(-max(max(lens), 1) // page) + 2) * page, dtype, window)


def cross_plan(c, dtype):
    B, T, S, Hq, Hk, Dh = c[:6]
    return attn_plan(B, T, Hq, Hk, Dh, S, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cases_take_the_forms_that_they_are_for(dtype):
    """On 256 units: a rule that moves leaves no form of a kernel untested."""
    for c in forms.TILES:
        assert paged_plan(c, dtype)[0] == "tiles", c
    assert {paged_plan(c, dtype)[1] for c in forms.TILES} >= {1, 2}
    for c in forms.TILE_PARTS:
        form, parts = paged_plan(c, dtype)[:2]
        assert form == "tiles" and parts > 4, c
    assert paged_plan(forms.TILE_PARTS[2], dtype)[1] > 512 // (3 * 16 * 4)  # more than two workgroups a unit
    assert all(paged_plan(c, dtype)[1] > 64 for c in forms.MANY_PARTS)
    assert {paged_plan(c, dtype)[0] for c in forms.MANY_PARTS} == {"rows", "steps"} | ({"tiles"} if dtype == "bf16" else set())
    for c in forms.TILE_CROSS:
        assert cross_plan(c, dtype)[0] == "tiles" and cross_plan(c, dtype)[1] < 3, c
    assert [cross_plan(c, dtype)[3] for c in forms.TILE_CROSS].count(True) == 1  # sorted
    for c in forms.TILE_CROSS_PARTS:
        form, parts = cross_plan(c, dtype)[:2]
        assert form == "tiles" and parts > 8, c
    for B, S, Hq, Hk, Dh, L, window in forms.UNSEEN + forms.UNSEEN_PARTS:
        form, parts = attn_plan(B, S, Hq, Hk, Dh, -(-L // 16) * 16, dtype, window)[:2]
        assert form == "tiles" and (parts > 8) == ((B, S, Hq, Hk, Dh, L, window) in forms.UNSEEN_PARTS)
    for Dh in (64, 128, 192):
        assert attn_plan(8, 300, 16, 16, Dh, 19 * 16, dtype)[0] == attn_plan(8, 300, 16, 16, Dh, 100, dtype)[0] == "tiles"
    B, S, Hq, Hk, Dh, _ = forms.FAR
    assert attn_plan(B, S, Hq, Hk, Dh, 1024, dtype)[0] == "tiles"
    got = {attn_plan(B, S, Hq, Hk, Dh, -(-L // 16) * 16, dtype)[:2] for B, S, Hq, Hk, Dh, L in edges.SIZES}
    for form in ("rows", "steps", "tiles"):  # each whole and in parts
        assert any(f == form and n == 1 for f, n in got) and any(f == form and n > 1 for f, n in got), form
    for cases, want in ((forms.APPEND_STREAM, (4, True)), (forms.APPEND_16, (16, False)), (forms.APPEND_4, (4, False))):
        for c in cases:
            assert append_form(*c[:5], dtype) == want, c
    assert append_form(*forms.APPEND_STREAM[0][:5], dtype, aligned=False) == (4, False)
    assert append_form(2, 7, 6, 3, 40, dtype) == (1, False)
