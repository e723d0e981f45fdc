"""The binding's view of a cache's memory: tensors that cannot hold the pages, or hold them in another order, are refused."""
import pytest
import torch

from paper_2602_06694_amd import binding as nq

pytestmark = pytest.mark.gpu

HEADS, PAGE, DIM, PAGES = 2, 16, 64, 5


def create(k, v, pages=PAGES, strides=(0, 0, 0)):
    nq.nq_kv_destroy(nq.nq_kv_create(k, v, nq.NQ_BF16, HEADS, DIM, PAGE, pages, *strides))


def memory(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")


def test_tensors_that_hold_the_pages():
    k, v = memory(PAGES, HEADS, PAGE, DIM), memory(PAGES, HEADS, PAGE, DIM)
    create(k, v)
    create(k, v, pages=1)
    create(k.view(-1), v)
    both = memory(3, 2, PAGES, HEADS, PAGE, DIM)
    create(both[1, 0], both[1, 1])
    wide = memory(PAGES, PAGE, HEADS * (DIM + 8))                      # slots before heads, rows with a gap
    strides = (PAGE * HEADS * (DIM + 8), HEADS * (DIM + 8), DIM + 8)
    create(wide, wide.clone(), strides=strides)
    create(wide[..., :HEADS * (DIM + 8) - 8], wide, strides=strides)    # (a view that ends with the last element)
    turned = memory(PAGES, PAGE, HEADS, DIM).transpose(1, 2)
    create(turned, turned.clone(memory_format=torch.preserve_format), strides=(turned.stride(0), turned.stride(2), turned.stride(1)))


@pytest.mark.parametrize("which", ["k", "v"])
def test_tensors_that_do_not(which):
    good = memory(PAGES, HEADS, PAGE, DIM)
    pair = lambda t: (t, good) if which == "k" else (good, t)  # noqa: E731
    for bad in (memory(PAGES - 1, HEADS, PAGE, DIM),                    # a page short
                memory(PAGES, HEADS, PAGE, DIM).view(-1)[:-8],
                memory(PAGES, PAGE, HEADS, DIM).transpose(1, 2),        # another order
                memory(1, HEADS, PAGE, DIM).expand(PAGES, -1, -1, -1)):  # one page, five times
        with pytest.raises(ValueError):
            create(*pair(bad))
    with pytest.raises(nq.NQError):                                     # (an empty tensor's address is NULL)
        create(*pair(memory(0)))
    with pytest.raises(ValueError):
        create(*pair(good), pages=PAGES + 1)
    with pytest.raises(ValueError):                                     # the last page's rows reach beyond
        create(*pair(memory(PAGES, HEADS, PAGE, DIM)), strides=(HEADS * (PAGE * DIM + 8), DIM, PAGE * DIM + 8))
    with pytest.raises(nq.NQError):                                     # what the library refuses it still does
        create(*pair(good), strides=(8, 8, 8))
