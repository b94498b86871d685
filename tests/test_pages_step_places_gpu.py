"""A step of more places than any model's: the most that n_tokens, an int32, can say."""
import pytest
import torch

import q4_ref as ref
from test_paged_gpu import I32, _ints, st  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("places", [2 ** 31 - 1, 2 ** 31 - 255, 2 ** 31 - 256])
def test_as_many_places_as_an_int_holds(st, places):
    table, lens, free = [[-1] * 9 for _ in range(3)], [0, 0, 0], list(range(20))
    d = [_ints(x) for x in (table, lens, [0] * 4, free, [20])]
    pt = st.make_pages(20, 16, *d[:3])
    slot = torch.full((places,), 5, dtype=I32, device="cuda")
    st.stlite_pages_step(pt, None, _ints([100, 0, 77]), d[3], d[4], slot)
    cu, n_free, want = ref.step(table, lens, None, [100, 0, 77], free, 20, 20, 16, 200)
    assert [x.tolist() for x in d] == [table, lens, cu, free, [n_free]]
    assert slot[:200].tolist() == want and int(slot[200:].max()) == int(slot[200:].min()) == -1
