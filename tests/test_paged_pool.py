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
