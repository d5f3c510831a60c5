"""PagedCache.read into rows that lie on each other is refused before anything is written; rows that interleave are taken."""
import pytest

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("kv", ["i8", "f32"])
def test_outputs_that_lie_on_each_other_are_refused(kv):
    import torch
    from paper_2503_08524_amd import D3Error, PagedCache
    cache = PagedCache(2, 2, 64, 4, 16, 1, 1, kv_dtype=kv, n_layers=2, device=DEV)
    slots = torch.arange(5, dtype=torch.int32, device=DEV)
    cache.append(0, slots, *(torch.randn(2, 5, 2, 64, device=DEV) for _ in range(2)))
    want = cache.read(0, slots, n_layers=2)
    buf = torch.full((4000,), 7.0, device=DEV)

    def rows(at, *strides):                                 # two layers of five rows of two heads: strides of layer, row and head
        return buf[at:].as_strided((2, 5, 2, 64), (*strides, 1))
    for strides, at in (((0, 128, 64), 2000), ((640, 0, 64), 2000), ((640, 128, 0), 2000),          # a dim whose entries are one
                        ((640, 128, 60), 2000), ((636, 128, 64), 2000),                             # rows that end in the next ones
                        ((640, 128, 64), 0), ((640, 128, 64), 32), ((640, 128, 64), 640), ((1280, 256, 64), 64)):       # k's and v's
        for k, v in ((rows(0, *strides), rows(at, *strides)), (rows(at, *strides), rows(0, *strides))):
            with pytest.raises(D3Error) as e:
                cache.read(0, slots, k, v)
            assert e.value.status == -1 and "lie on each other" in str(e.value) and (buf == 7).all()
    # side by side: a head's k and v, a row's, a layer's, all of them; in other orders of the dims
    for strides, at in (((1280, 256, 128), 64), ((1280, 256, 64), 128), ((1280, 128, 64), 640), ((640, 128, 64), 1280), ((64, 128, 1280), 640), ((64, 128, 640), 1408), ((640, 64, 320), 2000)):
        for k, v in ((rows(0, *strides), rows(at, *strides)), (rows(at, *strides), rows(0, *strides))):
            cache.read(0, slots, k, v)
            assert torch.equal(k, want[0]) and torch.equal(v, want[1]) and int((buf == 7).sum()) == 4000 - 2 * 1280
            buf.fill_(7)
    # a stride of a dim with one entry says nothing
    k, v = cache.read(1, slots[:1], buf.as_strided((1, 2, 64), (0, 64, 1)), buf[128:].as_strided((1, 2, 64), (0, 64, 1)))
    assert torch.equal(k[0], want[0][1, 0]) and torch.equal(v[0], want[1][1, 0])
