"""The linear layers' workspace may start on any 16-byte boundary, though the pieces of sums in it move 32 bytes at a time."""
import ctypes as C

import pytest
import torch

import test_training_cpu as host
from paper_2506_17974_b200 import binding as B
from paper_2506_17974_b200 import training as tr

lib = host.lib
PRODUCTS = ["forward", "grad_input", "grad_weight"]


def sizes(product):
    return dict(forward=(64, 1 << 16, 128), grad_input=(64, 128, 1 << 16), grad_weight=(1 << 16, 128, 64))[product]


def arguments(product, **at):
    rows, cin, cout = sizes(product)
    return host.linear(rows=rows, cin=cin, cout=cout, ld_x=cin, ld_w=cin, ld_dz=cout, ld_out=cout if product == "forward" else cin, **at)


@pytest.mark.parametrize("product", PRODUCTS)
def test_room_to_align_the_pieces(lib, product):
    """Pieces are whole tiles of 128 x 128 fp32 values, so what the library asks for beyond a multiple of one is the room in which
    their start can move from a 16-byte to a 32-byte boundary."""
    need = C.c_size_t(0)
    assert lib.lqsgd_linear_workspace_bytes(PRODUCTS.index(product), C.byref(arguments(product)), C.byref(need)) == 0
    assert need.value > 128 * 128 * 4 and need.value % (128 * 128 * 4) >= 16


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("product", PRODUCTS)
@pytest.mark.parametrize("offset", [16, 32, 48])
def test_workspace_on_any_16_byte_boundary(lib, product, offset, dtype):
    rows, cin, cout = sizes(product)
    g = torch.Generator("cuda").manual_seed(1)
    x, w, dz = (torch.randn(*s, generator=g, device="cuda").mul_(0.1).to(dtype) for s in ((rows, cin), (cout, cin), (rows, cout)))
    if product == "forward":
        want = tr.linear(x, w).y
    else:
        want = tr.linear_grad_input(dz, w) if product == "grad_input" else tr.linear_grad_weight(dz, x)
    out = torch.zeros_like(want)
    a = arguments(product, dtype=tr.DTYPES[dtype], x=x.data_ptr(), w=w.data_ptr(), dz=dz.data_ptr(), out=out.data_ptr())
    need = C.c_size_t(0)
    assert lib.lqsgd_linear_workspace_bytes(PRODUCTS.index(product), C.byref(a), C.byref(need)) == 0
    held = torch.full((need.value + offset + 64,), 0x5a, dtype=torch.uint8, device="cuda")
    assert held.data_ptr() % 256 == 0
    a.workspace, a.workspace_bytes = held.data_ptr() + offset, need.value
    assert getattr(lib, "lqsgd_linear_" + product)(C.byref(a), C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    assert (held[:offset] == 0x5a).all() and (held[offset + need.value:] == 0x5a).all()
    a.workspace = held.data_ptr() + 8
    assert getattr(lib, "lqsgd_linear_" + product)(C.byref(a), None) == B.ERR_MISALIGNED
