"""Bounded waits of the products of rows of codes: one that runs out returns, says so in the status word, and the next product is as if nothing had been."""
import ctypes as C
import time

import pytest
import torch

import test_training_rows_cpu as host
from paper_2506_17974_b200 import binding as B

lib = host.lib
LOADER, SECOND, MMA = 1, 2, 3
LIMIT = 4096                                    # polls of about a microsecond; no wait of these products is near it
# One of each way to deal the work out: k blocks of 128 terms that the first cluster has, whether a cluster is a pair of SMs.
CASES = [  # rows, in, out, k blocks, pair
    (4096, 1024, 4096, 32, True),                            # whole tiles of 256 x 256, several to a pair
    (1300, 131056, 130, 84, True),                           # long sums in equal shares
    (1024, 1024, 1024, 8, False),                            # whole tiles of 128 x 128
    (40, 4096, 640, 4, False),                               # the CTAs of a cluster sum one tile together
    (40, 16384, 128, 4, False),                              # one tile in equal shares
]


class Product:
    def __init__(self, lib, rows, cin, cout):
        g = torch.Generator("cuda").manual_seed(1)
        self.x, self.w = (torch.randint(-127, 128, (r, cin), generator=g, device="cuda", dtype=torch.int8) for r in (rows, cout))
        self.sx, self.sw = (torch.full((n,), 0.01, device="cuda") for n in (rows, cout))
        self.out = torch.empty(rows, cout, device="cuda", dtype=torch.bfloat16)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.call = lib.lqsgd_linear_rows8_forward
        self.a = host.linear8(rows=rows, cin=cin, cout=cout, x=host.Rows8(self.x.data_ptr(), cin, self.sx.data_ptr()),
                              w=host.Rows8(self.w.data_ptr(), cin, self.sw.data_ptr()), out=self.out.data_ptr(), ld_out=cout, status=self.status.data_ptr())
        need = C.c_size_t(0)
        assert lib.lqsgd_linear_rows8_workspace_bytes(C.byref(self.a), C.byref(need)) == 0
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
@pytest.mark.parametrize("rows,cin,cout,blocks,pair", CASES)
def test_a_wait_that_runs_out_is_reported_and_leaves_nothing_behind(lib, rows, cin, cout, blocks, pair):
    p = Product(lib, rows, cin, cout)
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
def test_a_product_by_dot_products_takes_the_stop_with_it(lib):
    """Two rows need no waits; what was armed for the call does not reach the next one."""
    few, many = Product(lib, 2, 512, 300), Product(lib, 40, 4096, 640)
    want, _ = many.run()
    assert lib.lqsgd_test_linear_wait(C.c_int32(MMA), C.c_int32(0), C.c_uint32(LIMIT)) == 0
    assert few.run()[1] == 0
    got, status = many.run()
    assert status == 0 and torch.equal(got, want)
