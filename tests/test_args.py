"""The compiled checks of tensor arguments (csrc/args.cpp), on the host: what they let through, with its pointer, and what they refuse.  (A CPU
tensor's device index is -1.)"""
import pytest
import torch

from paper_2605_23200_amd import binding as B

CPU = -1


@pytest.fixture(autouse=True)
def loaded():
    B.lib()


def test_pointer_of_what_fits():
    t = torch.zeros((3, 4), dtype=torch.int32)
    assert B._arg(t, torch.int32, 12, CPU, "t") == t.data_ptr()
    assert B._arg(t, torch.int32, 0, CPU, "t") == t.data_ptr()
    assert B._arg(t[1:], torch.int32, 8, CPU, "t") == t.data_ptr() + 16
    assert B._arg(t[:, :1][:1], torch.int32, 1, CPU, "t") == t.data_ptr()            # strides of extents of one
    assert B._arg(torch.nn.Parameter(torch.zeros(3)), torch.float32, 3, CPU, "t")
    assert B._arg(None, torch.int32, 12, CPU, "t") is None


@pytest.mark.parametrize("t", [torch.zeros(11, dtype=torch.int32), torch.zeros(12), torch.zeros(12, dtype=torch.int64), 7, "x", [1],
                               torch.zeros((4, 6), dtype=torch.int32)[:, ::2], torch.zeros((3, 4), dtype=torch.int32).t(),
                               torch.zeros((3, 4), dtype=torch.int32).to_sparse()])
def test_refused_with_its_name(t):
    with pytest.raises(ValueError, match="lens: contiguous torch.int32 tensor of at least 12 elements on GPU -1 expected"):
        B._arg(t, torch.int32, 12, CPU, "lens")


def test_another_device_and_no_type():
    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="on GPU 0 expected"):
        B._arg(t, torch.int32, 4, 0, "t")
    with pytest.raises(ValueError):
        B._arg(t, "int32", 4, CPU, "t")
    with pytest.raises(TypeError):
        B._arg(t, torch.int32, "4", CPU, "t")
    with pytest.raises(TypeError):
        B._arg(t, torch.int32, 4, CPU)


def test_rows_of_tokens():
    x = torch.zeros((2, 3, 4, 10 * 64 + 16))
    v = x[..., :640].unflatten(-1, (10, 64))
    assert B._token_rows(v[..., 2:5, :], (2, 3, 4, 3, 64), torch.float32, CPU, "k") == (x.data_ptr() + 2 * 64 * 4, 656)
    one = torch.zeros((1, 1, 1, 3, 64))
    assert B._token_rows(one, (1, 1, 1, 3, 64), torch.float32, CPU, "k") == (one.data_ptr(), 192)
    assert B._token_rows(x[:, :, :1, :64].unflatten(-1, (1, 64)), (2, 3, 1, 1, 64), torch.float32, CPU, "k")[1] == 4 * 656


@pytest.mark.parametrize("bad", [lambda v: v[..., ::2], lambda v: v[..., ::2, :], lambda v: v.double(), lambda v: v[0], lambda v: v[:, :2],
                                 lambda v: v.transpose(1, 2), lambda v: v.numpy(), lambda v: None])
def test_rows_that_do_not_fit(bad):
    v = torch.zeros((2, 3, 3, 6, 64))
    with pytest.raises(ValueError):
        B._token_rows(bad(v), (2, 3, 3, 6, 64), torch.float32, CPU, "k")


def test_one_stride_from_token_to_token():
    x = torch.zeros((2, 4, 4, 3, 64))
    for v, shape in ((x[:, :3], (2, 3, 4, 3, 64)), (x[:, :, :3], (2, 4, 3, 3, 64)), (x[:, :, ::2], (2, 4, 2, 3, 64))):
        if v.stride(2) * v.shape[2] == v.stride(1) and v.stride(1) * v.shape[1] == v.stride(0):
            continue
        with pytest.raises(ValueError, match="one stride"):
            B._token_rows(v, shape, torch.float32, CPU, "k")


def _nested(shape):
    import warnings
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")
        return torch.nested.nested_tensor([torch.zeros(shape), torch.zeros((1,) + shape[1:])])


def test_tensors_without_memory_of_their_own_are_refused():
    """Asked for their sizes or their memory, these throw, or answer with none: an error here, not the end of the process."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    shape = (2, 2, 2, 1, 64)
    with FakeTensorMode():
        fake = torch.zeros(shape)
    refused = []

    def both(t):
        for call in (lambda: B._arg(t, torch.float32, 4, CPU, "t"), lambda: B._token_rows(t, shape, torch.float32, CPU, "t")):
            with pytest.raises(ValueError, match="expected"):
                call()
            refused.append(1)
        return t

    both(fake)
    both(torch.zeros(shape, device="meta"))
    both(_nested(shape[1:]))
    torch.vmap(both)(torch.zeros((3,) + shape))
    assert len(refused) == 8
    assert B._arg(torch.zeros(0), torch.float32, 0, CPU, "t") == 0
