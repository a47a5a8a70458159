"""The path that a bounded wait of a linear product takes when it runs out: a role of the first cluster stops early, the kernel returns,
the status word says so, and the next product is as if nothing had been."""
import ctypes as C
import time

import pytest
import torch

import test_training_cpu as host
from paper_2506_17974_b200 import binding as B
from paper_2506_17974_b200 import training as tr

lib = host.lib
PRODUCTS = ["forward", "grad_input", "grad_weight"]
LOADER, SECOND, MMA = 1, 2, 3
LIMIT = 4096                                    # polls of about a microsecond; no wait of these products is near it
# One of each way to deal the work out: k blocks of 64 terms that the first cluster has, whether a cluster is a pair of SMs.
CASES = [  # product, rows, in, out, k blocks, pair
    ("forward", 4096, 512, 4096, 24, True),                  # whole tiles of 256 x 256, several to a pair
    ("grad_input", 4096, 4096, 512, 24, True),
    ("grad_weight", 16384, 2304, 2304, 280, True),           # long sums in equal shares, several accumulators to a tile
    ("forward", 1024, 256, 1024, 4, False),                  # whole tiles of 128 x 128
    ("forward", 256, 3136, 512, 7, False),                   # the CTAs of a cluster sum one tile together
    ("grad_weight", 8192, 512, 512, 16, False),
    ("grad_weight", 65536, 64, 128, 7, False),               # one tile in equal shares
]


def test_arming_refuses_what_it_does_not_know(lib):
    for role, after, limit in ((0, 0, 256), (4, 0, 256), (LOADER, -1, 256), (LOADER, 0, 15), (LOADER, 0, (1 << 18) + 1)):
        assert lib.lqsgd_test_linear_wait(C.c_int32(role), C.c_int32(after), C.c_uint32(limit)) == B.ERR_INVALID_ARG


class Product:
    def __init__(self, lib, product, rows, cin, cout):
        g = torch.Generator("cuda").manual_seed(1)
        self.x, self.w, self.dz = (torch.randn(*s, generator=g, device="cuda").mul_(0.1).bfloat16() for s in ((rows, cin), (cout, cin), (rows, cout)))
        shape = dict(forward=(rows, cout), grad_input=(rows, cin), grad_weight=(cout, cin))[product]
        self.out = torch.empty(shape, device="cuda", dtype=torch.float32 if product == "grad_weight" else torch.bfloat16)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.call = getattr(lib, "lqsgd_linear_" + product)
        self.a = host.linear(rows=rows, cin=cin, cout=cout, x=self.x.data_ptr(), ld_x=cin, w=self.w.data_ptr(), ld_w=cin, dz=self.dz.data_ptr(),
                             ld_dz=cout, out=self.out.data_ptr(), ld_out=shape[1], status=self.status.data_ptr())
        need = C.c_size_t(0)
        assert lib.lqsgd_linear_workspace_bytes(PRODUCTS.index(product), C.byref(self.a), C.byref(need)) == 0
        self.workspace = torch.zeros(max(1, need.value), dtype=torch.uint8, device="cuda")
        self.a.workspace, self.a.workspace_bytes = self.workspace.data_ptr(), need.value

    def run(self):
        """(output, status) of a call."""
        self.out.zero_()
        self.status.zero_()
        assert self.call(C.byref(self.a), C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
        torch.cuda.synchronize()
        return self.out.clone(), int(self.status.item())


@pytest.mark.gpu
@pytest.mark.parametrize("product,rows,cin,cout,blocks,pair", CASES)
def test_a_wait_that_runs_out_is_reported_and_leaves_nothing_behind(lib, product, rows, cin, cout, blocks, pair):
    p = Product(lib, product, rows, cin, cout)
    want, status = p.run()
    assert status == 0
    for role in (LOADER, SECOND, MMA):
        for after in sorted({0, 1, 3, blocks // 2, blocks - 1}):
            start = time.time()
            assert lib.lqsgd_test_linear_wait(C.c_int32(role), C.c_int32(after), C.c_uint32(LIMIT)) == 0
            got, status = p.run()
            assert time.time() - start < 10
            if role == SECOND and not pair:                  # nobody has that role
                assert status == 0 and torch.equal(got, want)
            else:
                assert status == B.STATUS_TIMEOUT, (role, after)
            for _ in range(2):                               # the next products: nothing armed, nothing left behind
                got, status = p.run()
                assert status == 0 and torch.equal(got, want), (role, after)


@pytest.mark.gpu
def test_a_stop_behind_the_last_k_block_is_none(lib):
    for product, rows, cin, cout, blocks, _ in CASES:
        p = Product(lib, product, rows, cin, cout)
        want, _ = p.run()
        assert lib.lqsgd_test_linear_wait(C.c_int32(MMA), C.c_int32(1 << 20), C.c_uint32(LIMIT)) == 0
        got, status = p.run()
        assert status == 0 and torch.equal(got, want)
