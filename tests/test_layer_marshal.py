"""What the calls of a serving step ask for and refuse before they touch a GPU: tensors without memory, no GPU."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
BF16, F32, I32, F8, U8 = torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn, torch.uint8


def tensors(device="cuda:0", **shapes):
    with FakeTensorMode():
        return {name: torch.empty(*shape, dtype=dtype, device=device) for name, (dtype, *shape) in shapes.items()}


# arguments of each call that fit, and those that are looked at last
CALLS = {
    "route": (dict(logits=(F32, 4, 8), expert=(I32, 8), weight=(F32, 8), offset=(I32, 9), source=(I32, 8), place=(I32, 8)), ["expert", "weight", "offset", "source", "place"],
              lambda t: (t["logits"], 2, t["expert"], t["weight"], t["offset"], t["source"], t["place"], None)),
    "combine": (dict(z=(BF16, 8, 16), place=(I32, 4, 2), y=(BF16, 4, 16), weight=(F32, 8), residual=(BF16, 4, 16)), ["weight"],
                lambda t: (t["z"], t["place"], t["y"], t["weight"], t["residual"])),
    "grouped_gemm": (dict(x=(BF16, 6, 32), w=(BF16, 2, 16, 32), offset=(I32, 3), y=(BF16, 6, 16), source=(I32, 6)), ["offset", "source"],
                     lambda t: (t["x"], t["w"], t["offset"], t["y"], t["source"])),
    "quantise": (dict(x=(BF16, 6, 32), q=(F8, 6, 32), scale=(F32, 6, 1)), ["scale"], lambda t: (t["x"], t["q"], t["scale"], 1)),
    "gemm_f8": (dict(x=(F8, 6, 32), xs=(F32, 6, 1), w=(U8, 16, 32), ws=(F32, 1, 1), y=(BF16, 6, 16)), ["xs", "ws"],
                lambda t: (t["x"], t["xs"], t["w"], t["ws"], t["y"], 128)),
    "grouped_gemm_f8": (dict(x=(F8, 6, 32), xs=(F32, 6, 1), w=(F8, 2, 16, 32), ws=(F32, 2, 1, 1), offset=(I32, 3), y=(BF16, 6, 16), source=(I32, 6)), ["offset", "source"],
                        lambda t: (t["x"], t["xs"], t["w"], t["ws"], t["offset"], t["y"], 128, t["source"])),
    "rmsnorm": (dict(x=(BF16, 6, 32), gain=(BF16, 32), residual=(BF16, 6, 32), h=(BF16, 6, 32), y=(BF16, 6, 32), q=(F8, 6, 32), scale=(F32, 6, 1), rstd=(F32, 6)), ["rstd"],
                lambda t: (t["x"], t["gain"], 1e-6, t["residual"], t["h"], t["y"], t["q"], t["scale"], t["rstd"])),
}


class StreamAsked(Exception):
    pass


@pytest.fixture
def native():
    module = B._native()

    def asked():
        raise StreamAsked

    module.set_current_stream(asked)
    yield module
    module.set_current_stream(lambda: B._stream(None))


@pytest.mark.parametrize("call", CALLS)
def test_the_stream_is_asked_for_last(native, call):
    shapes, last, arguments = CALLS[call]
    with pytest.raises(StreamAsked):                # everything fits
        getattr(native, call)(*arguments(tensors(**shapes)), None)
    for name in last:
        dtype, *shape = shapes[name]
        short = shapes | {name: (dtype, *shape[:-1], shape[-1] - 1)}
        with pytest.raises(ValueError):
            getattr(native, call)(*arguments(tensors(**short)), None)


# the calls that binding.py takes apart itself
BACKWARD = {
    "csr5_route_backward": dict(expert=(I32, 4, 2), weight=(F32, 4, 2), dweight=(F32, 4, 2), dlogits=(BF16, 4, 8)),
    "csr5_combine_backward": dict(dy=(BF16, 4, 16), z=(BF16, 8, 16), place=(I32, 4, 2), weight=(F32, 4, 2), dz=(BF16, 8, 16), dweight=(F32, 4, 2)),
    "csr5_grouped_gemm_dx": dict(dy=(BF16, 6, 16), w=(BF16, 2, 16, 32), offset=(I32, 3), dx=(BF16, 6, 32)),
    "csr5_grouped_gemm_dw": dict(dy=(BF16, 6, 16), x=(BF16, 6, 32), offset=(I32, 3), dw=(BF16, 2, 16, 32), source=(I32, 6)),
    "csr5_rmsnorm_backward": dict(h=(BF16, 6, 32), gain=(BF16, 32), rstd=(F32, 6), dy=(BF16, 6, 32), dh=(BF16, 6, 32), dgain=(F32, 32), workspace=(U8, 4096),
                                  residual_grad=(BF16, 6, 32)),
}


class Stream:
    cuda_stream = 4096

    def __init__(self, gpu):
        self.device_index = gpu


@pytest.mark.parametrize("call", CALLS)
def test_tensors_of_several_gpus_are_refused(native, call):
    shapes, _, arguments = CALLS[call]
    here = tensors(**shapes)
    for name, shape in shapes.items():
        with pytest.raises(ValueError, match="GPU"):
            getattr(native, call)(*arguments(here | tensors("cuda:1", **{name: shape})), None)
    with pytest.raises(ValueError, match="stream is one of GPU 1"):
        getattr(native, call)(*arguments(here), Stream(1))
    assert getattr(native, call)(*arguments(here), Stream(0)) == B.CSR5_EINVAL          # tensors without memory: the library's own refusal
    assert getattr(native, call)(*arguments(here), 4096) == B.CSR5_EINVAL


@pytest.mark.parametrize("call", BACKWARD)
def test_tensors_of_several_gpus_are_refused_backward(call):
    shapes = BACKWARD[call]
    here, run = tensors(**shapes), getattr(B, call)
    for name, shape in shapes.items():
        with pytest.raises(ValueError, match="GPU"):
            run(**(here | tensors("cuda:1", **{name: shape})), stream=Stream(0))
    with pytest.raises(ValueError, match="stream is one of GPU 1"):
        run(**here, stream=Stream(1))
    assert run(**here, stream=Stream(0), check=False) == B.CSR5_EINVAL
