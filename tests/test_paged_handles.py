"""The handles of the paged cache hold the addresses of their own tensors, however they come about, and only of tensors that the library
reads as what they are (no GPU)."""
import copy
import dataclasses
import io
import pickle

import pytest
import torch


@pytest.fixture(scope="module")
def F():
    from paper_2604_07394_amd import binding
    return binding


def made_anew(F, h):
    return type(h)(*(getattr(h, f.name) for f in dataclasses.fields(h)))


def saved(h):
    buf = io.BytesIO()
    torch.save(h, buf)
    buf.seek(0)
    return torch.load(buf, weights_only=False)               # (written three lines above)


@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda h: pickle.loads(pickle.dumps(h)), saved], ids=["copy", "deepcopy", "pickle", "save"])
@pytest.mark.parametrize("which", ["pages", "pool", "strided pool"])
def test_a_copy_holds_the_addresses_of_its_own_tensors(F, how, which):
    h = F.PageTable.empty(2, 3, 5, device="cpu") if which == "pages" else F.PagedKV.empty(3, 2, 64, device="cpu")
    if how is not copy.copy and which == "pool":             # (torch pickles tensors of uint8, but none of float8)
        h = F.PagedKV(h.k.view(torch.uint8), h.v.view(torch.uint8), h.k_scale, h.v_scale)
    if which == "strided pool":
        wide = torch.zeros(3, 2, 64, 112, dtype=torch.uint8)
        h = F.PagedKV(wide[..., 16:80], wide.clone()[..., 16:80], h.k_scale, h.v_scale)
    c = how(h)
    assert type(c) is type(h) and c.packed == made_anew(F, c).packed
    first = dataclasses.fields(h)[0].name
    assert (getattr(c, first).data_ptr() == getattr(h, first).data_ptr()) == (how is copy.copy) == (c.packed == h.packed)


@pytest.mark.parametrize("dtype", [d for d in ("float8_e4m3fnuz", "float8_e5m2", "float8_e5m2fnuz", "int8", "bool") if hasattr(torch, d)])
def test_codes_of_another_type_are_refused(F, dtype):
    """Types of one byte whose codes stand for other values: read as e4m3 they would give wrong results without a word."""
    good = F.PagedKV.empty(3, 2, 64, device="cpu")
    k = torch.zeros(3, 2, 64, 64, dtype=torch.uint8).view(getattr(torch, dtype))
    for pair in ((k, k.clone()), (good.k, k), (k, good.v)):
        with pytest.raises(AssertionError):
            F.PagedKV(*pair, good.k_scale, good.v_scale)
    F.PagedKV(good.k, good.v.view(torch.uint8), good.k_scale, good.v_scale)
