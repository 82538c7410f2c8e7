"""cp_token_sample on more rows than a grid's first dimension has workgroups for, with several draws each."""
import pytest
import torch

import paper_1711_01912_amd as cpe

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("V,G", [(9, 40), (16, 63)])
def test_workgroups_behind_the_last_row_draw_nothing(V, G):
    # 16 rows a workgroup, 2^22 workgroups in the first dimension: the second has up to 2^22 - 1 too many, for which (rows left) * G, a
    # number below -2^31, must not become one above 0
    rows, guard = 2 ** 26 + 3, 1 << 20
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.empty(rows, V, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    u = torch.rand(1, G, generator=g, device=DEV).expand(rows, G)
    room = torch.full((guard + rows * G + guard,), 99, dtype=torch.uint8, device=DEV)
    tokens = room[guard:-guard].view(rows, G)
    cpe.cp_token_sample(x, u, out={"tokens": tokens})
    assert bool((room[:guard] == 99).all()) and bool((room[-guard:] == 99).all())
    assert int(tokens.max()) < V
    for lo in (0, 2 ** 25 - 5, rows - 1000):
        part = cpe.cp_token_sample(x[lo:lo + 1000], u[lo:lo + 1000], dtype=torch.uint8)["tokens"]
        assert torch.equal(tokens[lo:lo + 1000], part), lo
