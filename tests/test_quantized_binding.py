"""What the binding of the narrow formats refuses before it calls the library, with stand-ins for tensors of several devices (no GPU needed)."""
import pytest
import torch

from paper_2506_12035_b200 import binding


class Tensor:
    """A contiguous tensor as far as the binding asks."""

    def __init__(self, dtype, *shape, device=0):
        self.dtype, self.shape, self.device_index, self.is_cuda = dtype, shape, device, device >= 0
        self.strides = tuple(int(torch.tensor(shape[i + 1:]).prod()) if i + 1 < len(shape) else 1 for i in range(len(shape)))

    def get_device(self):
        return self.device_index

    def is_contiguous(self):
        return True

    def numel(self):
        return int(torch.tensor(self.shape).prod())

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def storage_offset(self):
        return 0

    def data_ptr(self):
        return 0x10000


class Reached(Exception):
    pass


class Library:
    def __getattr__(self, name):
        def call(*args):
            raise Reached(name)
        return call


B, S, H, dh, n = 2, 64, 2, 64, 3
D = H * dh


def model():
    m = binding.Marche.__new__(binding.Marche)
    m.h, m.lib, m.device_index, m.operand_dtype, m.torch_dtype = None, Library(), 0, torch.float16, torch.bfloat16
    return m


def cache(codes=0, scales=0):
    return binding.QuantizedCache(Tensor(torch.int8, 2, B, S, D, device=codes), Tensor(torch.float32, 2, B, H, 64, device=scales), H)


def weights(codes=0, scales=0):
    return binding.QuantizedWeights(Tensor(torch.uint8, 32 * 128 // 2, device=codes), Tensor(torch.bfloat16, 32 * 2, device=scales), 32, 128, 64)


def rows(dtype=torch.bfloat16, device=0, width=D):
    return Tensor(dtype, B * n, width, device=device)


CALLS = {
    "scatter": lambda m, c=None, a=0, b=0, i=0, s=None: m.scatter_kv_quantized(rows(device=a), rows(device=b), D, Tensor(torch.int32, B, n, device=i), n, c or cache(), s),
    "gather": lambda m, c=None, a=0, b=0, i=0, s=None: m.gather_kv_quantized(c or cache(), Tensor(torch.int32, B, n, device=i), n, rows(device=a), rows(device=b), D, s),
    "attention": lambda m, c=None, a=0, b=0, i=0, s=None: m.attention_quantized(rows(device=a), D, n, H, c or cache(), Tensor(torch.int32, B, device=i),
                                                                               rows(torch.float16, device=b), s),
    "linear": lambda m, c=None, a=0, b=0, i=0, s=None: m.linear_quantized(rows(torch.float16, device=a), c or weights(), Tensor(torch.float32, 32, device=i), 2,
                                                                         rows(torch.float16, device=b, width=32), stream=s),
}


class Stream:
    cuda_stream = 0x20


@pytest.mark.parametrize("call", CALLS)
def test_tensors_of_another_device_are_refused(call):
    m = model()
    with pytest.raises(Reached):
        CALLS[call](m, s=Stream())
    for which in "abi":
        for device in (1, -1):
            with pytest.raises(AssertionError):
                CALLS[call](m, s=Stream(), **{which: device})
    with pytest.raises(AssertionError):                              # all of them on one device, but not the context's
        CALLS[call](m, c=weights(1, 1) if call == "linear" else cache(1, 1), a=1, b=1, i=1, s=Stream())
    with pytest.raises(AssertionError):
        m.device_index = 1
        CALLS[call](m, s=Stream())


@pytest.mark.parametrize("make", [cache, weights])
def test_codes_and_scales_are_on_one_device(make):
    for codes, scales in ((0, 1), (1, 0), (0, -1), (-1, 0)):
        with pytest.raises(AssertionError):
            make(codes, scales)


def test_a_matrix_of_another_device_is_not_laid_out():
    with pytest.raises(AssertionError):
        model().quantize_weights(Tensor(torch.float32, 32, 128, device=1), 64)
