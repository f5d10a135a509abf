"""What a page pool refuses before a kernel could see it (no GPU needed: the checks come before that for one)."""
import pytest
import torch

import paper_2502_17599_amd as pkg

TYPES = [torch.float32, torch.bfloat16, torch.uint8]


def _pages(dtype, n=5, heads=2, page=16, d=64):
    return torch.zeros((n, heads, page, d), dtype=dtype)


def _scales(dtype, n=5, heads=2, page=16):
    return [torch.zeros((n, heads, page)) for _ in range(2)] if dtype == torch.uint8 else []


@pytest.mark.parametrize("dtype", TYPES)
def test_pages_that_repeat_or_overlap_are_refused(dtype):
    """One page in memory that counts as five: the library would look for the others behind it."""
    k, v = (_pages(dtype, 1).expand(5, -1, -1, -1) for _ in range(2))
    with pytest.raises(ValueError, match="lie 0 apart"):
        pkg.PagePool(k, v, *_scales(dtype))
    size = 2 * 16 * 64
    for step in (16, size // 2, size - 16):
        k, v = (_pages(dtype).flatten().as_strided((5, 2, 16, 64), (step, 16 * 64, 64, 1)) for _ in range(2))
        with pytest.raises(ValueError, match=f"lie {step} apart"):
            pkg.PagePool(k, v, *_scales(dtype))


@pytest.mark.parametrize("dtype", TYPES)
def test_what_was_taken_still_is_up_to_the_device(dtype):
    """Pages next to each other, apart, K and V interleaved, a single page of any stride: all that is missing is the GPU."""
    both = torch.zeros((5, 2, 2, 16, 64), dtype=dtype)
    apart = torch.zeros((5, 3, 2, 16, 64), dtype=dtype)
    for k, v in ((_pages(dtype), _pages(dtype)), (both[:, 0], both[:, 1]), (apart[:, 2], apart[:, 0])):
        with pytest.raises(ValueError, match="on the GPU"):
            pkg.PagePool(k, v, *_scales(dtype))
    one = [_pages(dtype, 1).as_strided((1, 2, 16, 64), (0, 16 * 64, 64, 1)) for _ in range(2)]
    with pytest.raises(ValueError, match="on the GPU"):
        pkg.PagePool(*one, *_scales(dtype, 1))


@pytest.mark.parametrize("dtype", TYPES)
def test_k_and_v_pages_that_share_memory_are_refused(dtype):
    """A token's k and v would be written to the same place."""
    x, size = torch.zeros(20 * 2 * 16 * 64, dtype=dtype), 2 * 16 * 64

    def pages(first, step, n=5):
        return x[first:].as_strided((n, 2, 16, 64), (step, 16 * 64, 64, 1))
    scales = _scales(dtype)
    for k, v in ((pages(0, size), pages(0, size)), (pages(0, size), pages(size, size)), (pages(0, 3 * size), pages(2 * size + 16, 3 * size)),
                 (pages(size - 16, 2 * size), pages(0, 2 * size)), (pages(0, 3 * size), pages(6 * size, 3 * size)),
                 (pages(0, size, 1), pages(64, size, 1))):
        for a, b in ((k, v), (v, k)):
            with pytest.raises(ValueError, match="share memory"):
                pkg.PagePool(a, b, *_scales(dtype, k.shape[0]))
    for k, v in ((pages(0, size), pages(5 * size, size)), (pages(0, 3 * size), pages(2 * size, 3 * size)), (pages(0, size, 1), pages(size, size, 1))):
        for a, b in ((k, v), (v, k)):
            with pytest.raises(ValueError, match="on the GPU"):
                pkg.PagePool(a, b, *_scales(dtype, k.shape[0]))
    if scales:
        with pytest.raises(ValueError, match="share memory"):
            pkg.PagePool(_pages(dtype), _pages(dtype), scales[0], scales[0])
