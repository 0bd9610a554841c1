"""Lists that a caller puts together are checked before any kernel reads them: tensors that only say they are on a device stand in
for those of one, so no GPU is needed."""
import pytest

from paper_2601_21198_b200 import build

E, T, K = 3, 5, 2


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


class On:
    """A tensor that answers as one on device `index`."""

    def __init__(self, tensor, index=0):
        self._tensor, self._index = tensor, index

    def get_device(self):
        return self._index

    def __getattr__(self, name):
        return getattr(self._tensor, name)


def lists(**other):
    import torch
    of = dict(offsets=On(torch.zeros(E + 1, dtype=torch.int32)), order=On(torch.zeros(T * K, dtype=torch.int32)),
              place=On(torch.zeros(T, K, dtype=torch.int32)))
    of.update(other)
    return of


def test_lists_that_are_right(zb):
    g = zb.TokenGroups(n_experts=E, **lists())
    assert (g.tokens, g.k, g.rows, g.n_experts, g.index) == (T, K, T * K, E, 0)


@pytest.mark.parametrize("name", ["offsets", "order", "place"])
def test_lists_of_another_type_place_or_density(zb, name):
    import torch
    right = lists()[name]._tensor
    apart = torch.zeros(*right.shape[:-1], 2 * right.shape[-1], dtype=torch.int32)[..., ::2]
    for wrong in (On(right.long()), On(right.float()), right, On(right, 1), On(apart), On(right[:-1]), On(right[None]), On(right.flatten()[:0])):
        with pytest.raises(ValueError):
            zb.TokenGroups(n_experts=E, **lists(**{name: wrong}))


def test_too_few_offsets_for_the_groups(zb):
    for n in (E - 1, E + 1):
        with pytest.raises(ValueError):
            zb.TokenGroups(n_experts=n, **lists())
