"""The cache's reordering over several layers: all of them, or, where one is refused, none."""

import pytest
import torch

from tests._decode import gen

pytestmark = pytest.mark.gpu

B = torch.bfloat16


@pytest.fixture(scope="module")
def de():
    assert torch.cuda.is_available()
    from paper_2307_04963_amd import decoding
    return decoding


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def layer(de, g, pages=12, heads=2, page=8, dim=16):
    return de.Cache(*(torch.randn((pages, heads, page, dim), generator=g, device="cuda").to(B) for _ in range(2)))


def unaligned(de, like):
    wide = [torch.zeros(t.numel() + 8, dtype=B, device="cuda") for t in like]
    return de.Cache(*(w[4:4 + t.numel()].view(t.shape) for w, t in zip(wide, like)))


def test_refused_layers(de):
    """A later layer that is refused leaves the earlier ones, the tables and the lengths as they are."""
    from paper_2307_04963_amd._lib import DyclError
    g = gen(1)
    first = layer(de, g)
    tables, lengths = ints(0, 1, 2, 3, 4, 5).view(2, 3), ints(13, 5)
    parents, fresh = ints(1, 0), ints(8, 9)
    bad = [de.Cache(*(t.float() for t in first)), de.Cache(first.keys, first.values[1:]), de.Cache(*(t.cpu() for t in first)),
           de.Cache(first.keys, None), de.Cache(*(t.transpose(1, 2) for t in first)), layer(de, g, page=16), layer(de, g, dim=20), layer(de, g, dim=264),
           layer(de, g, pages=0), de.Cache(first.keys, first.keys), unaligned(de, first)]
    for i, wrong in enumerate(bad):
        for layers in ([first, wrong], [first, layer(de, g), wrong]):
            before = [t.clone() for t in first]
            out_tables, out_lengths = torch.full((2, 3), 77, dtype=torch.int32, device="cuda"), ints(77, 77)
            with pytest.raises((ValueError, DyclError)):
                de.fork(layers, tables, lengths, parents, fresh, out_tables=out_tables, out_lengths=out_lengths)
                print("accepted:", i)
            assert all(torch.equal(a, b) for a, b in zip(first, before)), i
            assert bool((out_tables == 77).all()) and bool((out_lengths == 77).all()), i
    with pytest.raises(ValueError):
        de.fork([first, layer(de, g)], tables, lengths, parents, fresh, page=16)


def test_layers_of_other_shapes(de):
    """Layers share tables and the tokens of a page; heads, dims and the number of pages are their own.  Four layers are as one each."""
    g = gen(2)
    layers = [layer(de, g), layer(de, g, heads=5, dim=64), layer(de, g, pages=20), layer(de, g, heads=1, dim=256)]
    tables, lengths = ints(0, 1, 2, 3, 4, 5).view(2, 3), ints(13, 5)
    parents, fresh = ints(1, 0, 0), ints(8, 9, 10)
    alone = [de.Cache(*(t.clone() for t in c)) for c in layers]
    got = de.fork(layers, tables, lengths, parents, fresh)
    for c in alone:
        want = de.fork(c, tables, lengths, parents, fresh, page=8)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    for c, d in zip(layers, alone):
        assert all(torch.equal(a, b) for a, b in zip(c, d))
        assert torch.equal(c.keys[8, :, :5], c.keys[3, :, :5]) and torch.equal(c.values[9, :, :5], c.values[1, :, :5])
    assert got[0].tolist() == [[8, 4, 5], [0, 9, 2], [0, 10, 2]] and got[1].tolist() == [5, 13, 13]
    # no layers, tuples, generators
    for none in (None, [], ()):
        assert all(torch.equal(a, b) for a, b in zip(de.fork(none, tables, lengths, parents, fresh, page=8), got))
    assert all(torch.equal(a, b) for a, b in zip(de.fork((c for c in layers), tables, lengths, parents, fresh), got))
