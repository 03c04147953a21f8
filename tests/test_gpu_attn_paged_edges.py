"""abq_attn_paged where scores, weights or hidden tokens are out of the ordinary: infinite keys, scores of any size, tokens that a row does
not see, and every token of a long context for itself."""
import pytest
import torch

from serving_reference import Paged

pytestmark = pytest.mark.gpu


def run(abq, p, scale=None, **kw):
    cache, batch, q = p.device()
    return abq.abq_attn_paged(cache, batch, q, p.dim ** -0.5 if scale is None else scale, **kw).cpu().view(p.rows, p.heads_q, p.dim)


def place(p, s, t):
    """Page and offset of token t of sequence s."""
    return int(p.pages[s, t // p.page]), t % p.page


class Without(Paged):
    """Tokens whose weight is zero: the 64-bit form leaves them out."""
    out = ()

    def held(self, which, s, t):
        return None if (s, t) in self.out else super().held(which, s, t)


# ---- infinite keys ---------------------------------------------------------------------------------
@pytest.mark.parametrize("n", [1, 3, 40, 90])
@pytest.mark.parametrize("dim", [16, 48, 64, 80, 96, 112, 128, 144, 160, 256])
def test_a_key_whose_score_is_minus_infinity_has_no_weight(abq, dim, n):
    """In any column, the first eight (which stand in for the columns behind narrower heads) among them."""
    for column in (0, 7, 8, dim - 1):
        p = Without([(n, 70), (2, 11)], 4, 2, dim, 16, seed=dim + column)
        p.q.view(p.rows, 4, dim)[..., column] = 1.0 + torch.arange(p.rows)[:, None] % 3
        p.out = [(0, 0), (0, 5), (0, 40), (1, 3)]
        for s, t in p.out:
            page, o = place(p, s, t)
            p.cache[0][page, :, o, column] = -float("inf")
        y = run(abq, p)
        want, bound = p.attention(dim ** -0.5)
        assert ((y.double() - want).abs() <= bound).all(), column


@pytest.mark.parametrize("n", [1, 3, 40, 90])
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
def test_a_key_whose_score_is_infinite_makes_its_row_nan(abq, dim, n):
    p = Paged([(n, 70)], 4, 2, dim, 16, seed=dim)
    p.q.view(p.rows, 4, dim)[..., 1] = 1.0
    page, o = place(p, 0, 70 + n - 1)
    p.cache[0][page, 0, o, 1] = float("inf")
    y = run(abq, p)
    assert y[n - 1, :2].isnan().all() and y[n - 1, 2:].isfinite().all() and y[:n - 1].isfinite().all()
