"""The paged cache beside autograd: nothing is recorded, so tensors that need a gradient are refused, and memory that a
graph keeps for its backward pass is not overwritten unnoticed."""
import pytest
import torch

from paged_cases import DEV, make_pool, normal
from test_gpu_paged_rows import _cache
from test_gpu_rotary import _plan

pytestmark = pytest.mark.gpu

T, H, D = 5, 2, 64


def _inputs():
    import paper_2502_17599_amd as pkg
    pool = make_pool("f32", 8, H, 16, D)
    table = torch.zeros((T, 1), dtype=torch.int32, device=DEV)
    lens = torch.full((T,), 3, dtype=torch.int32, device=DEV)
    return (pool, _plan(D, 1, False, 0)[0], torch.arange(T, dtype=torch.int32, device=DEV), torch.arange(T, device=DEV), normal(1, T, H, D),
            table, lens, pkg.PagedDecoder(pool, T, H, 1))


def test_tensors_that_require_grad_are_refused():
    import paper_2502_17599_amd as pkg
    pool, rope, pos, slots, x, table, lens, dec = _inputs()
    leaf = x.clone().requires_grad_()
    made = leaf * 2                                      # not a leaf
    cc, _ = _cache([[5, 6]], H, D, "f32", False, 1)
    cc.v_out.requires_grad_()
    pages = pool.k_pages.clone()
    for g in (leaf, made):
        for call in (lambda: pkg.meda_rotary(g, None, pos, rope), lambda: pkg.meda_rotary(x, g, pos, rope), lambda: pkg.meda_rotary(g, None, pos, rope, g),
                     lambda: pkg.meda_rotary(x, None, pos, rope, g), lambda: pkg.meda_rotary(x, x, pos, rope, None, g),
                     lambda: pkg.meda_paged_append(pool, g, x, slots), lambda: pkg.meda_paged_append(pool, x, g, slots),
                     lambda: pkg.meda_paged_append(pool, x, x, slots, g), lambda: pkg.meda_paged_append(pool, x, x, slots, x, q_out=g),
                     lambda: dec(g, table, lens), lambda: dec(x, table, lens, g), lambda: pkg.meda_paged_store(pool, cc, table[:2], lens[:2])):
            with pytest.raises(ValueError, match="requires grad"):
                call()
    assert torch.equal(pool.k_pages, pages)
    with pytest.raises(ValueError, match="requires grad"):
        pkg.PagePool(pages.requires_grad_(), pool.v_pages)
    want = pkg.meda_rotary(x, x, pos, rope)[0]
    with torch.no_grad():                                # as a program that only answers runs
        assert torch.equal(pkg.meda_rotary(leaf, made, pos, rope)[0], want)
        assert torch.equal(dec(leaf, table, lens).clone(), dec(x, table, lens))
        pkg.meda_paged_append(pool, made, leaf, slots, leaf)
    with torch.inference_mode():
        assert torch.equal(pkg.meda_rotary(x * 1, None, pos, rope, x * 0)[0], want)
    assert torch.equal(pkg.meda_rotary(leaf.detach(), None, pos, rope)[0], want)


@pytest.mark.parametrize("how", ["in place", "k_out", "append", "out", "decoder's own"])
def test_what_a_graph_keeps_is_not_overwritten_unnoticed(how):
    import paper_2502_17599_amd as pkg
    pool, rope, pos, slots, x, table, lens, dec = _inputs()
    kept = dec(x, table, lens) if how == "decoder's own" else x.clone()
    w = torch.ones_like(x).requires_grad_()
    y = (w * kept).sum()                                 # keeps `kept` for w's gradient
    other = x * 3
    {"in place": lambda: pkg.meda_rotary(kept, None, pos, rope, kept), "k_out": lambda: pkg.meda_rotary(x, other, pos, rope, None, kept),
     "append": lambda: pkg.meda_paged_append(pool, x, x, slots, other, pos, rope, kept), "out": lambda: dec(other, table, lens, kept),
     "decoder's own": lambda: dec(other, table, lens)}[how]()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_gradient_by_the_inverse_matches_autograd():
    """dL/dx of L = <g, R x>: the inverse call against autograd through the same rotation in float64 (tolerance of one turn:
    tests of the rotation, 2^-20 of the pair)."""
    import paper_2502_17599_amd as pkg
    rope, freq, _ = _plan(D, 1, False, 0)
    pos = torch.tensor([0, 3, 77, 1234, 99999], dtype=torch.int32, device=DEV)
    x, g = normal(1, T, H, D), normal(2, T, H, D)
    with torch.no_grad():
        got = pkg.meda_rotary(g, None, pos, rope, inverse=True)[0]
    a = x.double().requires_grad_()
    angle = (pos.double()[:, None] * torch.from_numpy(freq).to(DEV))[:, None]
    first, second = a[..., :D // 2], a[..., D // 2:]
    y = torch.cat([first * angle.cos() - second * angle.sin(), second * angle.cos() + first * angle.sin()], -1)
    (y * g.double()).sum().backward()
    size = g.double().abs()
    pair = size + torch.roll(size, D // 2, -1)
    assert ((got.double() - a.grad).abs() <= 2.0 ** -20 * pair).all()
