"""An F8 and the memory that it stands for: what a call hands to the library is what the object shows (no GPU needed)."""
import pytest

torch = pytest.importorskip("torch")
from paper_1905_10830_amd import binding as fmtc  # noqa: E402


def _some(rows=4, depth=200, **more):
    return fmtc.f8_empty(rows, depth, device="cpu", **more)


@pytest.mark.parametrize("name", ["codes", "scales", "rows", "depth", "block_rows"])
def test_what_it_holds_is_not_assigned_anew(name):
    q = _some()
    before = getattr(q, name)
    with pytest.raises(AttributeError):
        setattr(q, name, _some(2).codes if name in ("codes", "scales") else 2)
    assert getattr(q, name) is before


def test_addresses_are_those_of_its_tensors():
    q = _some()
    c = fmtc._f8(q)._obj
    assert (c.d_codes, c.d_scales) == (q.codes.data_ptr(), q.scales.data_ptr())
    assert (c.rows, c.depth, c.ld, c.ld_scales) == (4, 200, 256, 4)
    assert fmtc._f8(None) is None
    fmtc._f8(_some(0))  # (no memory at all)


@pytest.mark.parametrize("which", ["codes", "scales"])
def test_a_tensor_that_went_elsewhere_is_refused(which):
    """`data` of a tensor can be exchanged under the object, and the memory it had before be freed."""
    q = _some()
    t = getattr(q, which)
    t.data = torch.empty_like(t)
    with pytest.raises(ValueError, match=which):
        fmtc._f8(q)


@pytest.mark.parametrize("which", ["codes", "scales"])
def test_a_tensor_that_grew_elsewhere_is_refused(which):
    q = _some()
    getattr(q, which).resize_(1 << 22)
    with pytest.raises(ValueError, match=which):
        fmtc._f8(q)
