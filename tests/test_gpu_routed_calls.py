"""The native calls of routing and of kept rows: where their results come from."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2104_08378_amd import sp24
from test_gpu_routed_block import Declines, calls, flat

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


class Sees(TorchDispatchMode):
    """Where the memory that torch hands out while it looks on begins."""

    def __init__(self):
        super().__init__()
        self.memory = set()

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        got = func(*args, **(kwargs or {}))
        if torch.is_tensor(got) and "empty" in func.__name__:
            self.memory.add(got.untyped_storage().data_ptr())
        return got


def test_a_dispatch_mode_sees_every_result():
    n = lambda *s: torch.randn(*s, device="cuda")  # noqa: E731
    x, w, l = n(64, 61).to(BF16), n(64, 64).to(BF16), n(64, 8)
    c, r = sp24.sp24_checkpoint_rows(x), sp24.sp24_moe_route(l, 2)
    offsets, slots, rows = sp24.sp24_moe_sort(r.ids, 8)
    dy = n(rows.numel(), 64).to(BF16)
    z = sp24.sp24_checkpoint_rows(dy)
    V, m = sp24.sp24_compress(w)
    new = [
        lambda: sp24.sp24_moe_route(l, 2, want_scores=True, want_load=True), lambda: sp24.sp24_moe_route_backward(l, r.ids, r.weights), lambda: sp24.sp24_checkpoint_rows(x),
        lambda: sp24.sp24_restore_rows(c, BF16), lambda: sp24.sp24_linear_backward_checkpoint(x, c, "relu"), lambda: sp24.sp24_linear_backward_checkpoint(dy, z, "gelu", offsets=offsets),
        lambda: sp24.sp24_gemm_dense_checkpoint(w.t(), c, BF16), lambda: sp24.sp24_gemm_dense_grouped_checkpoint(dy.t(), c, offsets, BF16, rows=rows, topk=2),
        lambda: sp24.sp24_compress(w), lambda: sp24.sp24_spmm(V, m, w, BF16), lambda: sp24.sp24_gemm_dense(w, w, BF16), lambda: sp24.sp24_prune(w),
        lambda: sp24.sp24_rmsnorm(w, torch.ones(64, device="cuda"), want_rstd=True)[0], lambda: sp24.sp24_quantize_rows(w, torch.int8), lambda: sp24.sp24_linear_backward(w, w, "silu"),
        lambda: sp24.sp24_moe_sort(r.ids, 8), lambda: sp24.sp24_moe_gather(w, rows, 2),
    ]
    for i, call in enumerate(new):
        with Sees() as mode:
            got = [t for t in flat(call()) if t is not None]
        assert got and all(t.untyped_storage().data_ptr() in mode.memory for t in got), i


@pytest.mark.parametrize("python_path", [False, True])
def test_new_memory_is_filled_where_torch_is_told_to(monkeypatch, python_path):
    """torch.use_deterministic_algorithms has new memory filled with NaN: the columns behind a padded result's."""
    if python_path:
        monkeypatch.setattr(sp24, "_host", Declines())
    g = torch.Generator(device="cuda").manual_seed(0)
    dy = torch.randn(48, 5, generator=g, device="cuda").to(BF16)
    z = sp24.sp24_checkpoint_rows(torch.randn(48, 5, generator=g, device="cuda"))
    want = sp24.sp24_linear_backward_checkpoint(dy, z, "gelu")
    torch.use_deterministic_algorithms(True)
    try:
        held = torch.zeros(48, 8, dtype=BF16, device="cuda")
        del held                                      # (what the allocator gives next holds zeros)
        dz, dzt, db = sp24.sp24_linear_backward_checkpoint(dy, z, "gelu")
    finally:
        torch.use_deterministic_algorithms(False)
    assert dz.stride() == (8, 1) and bool(torch.isnan(torch.as_strided(dz, (47, 3), (8, 1), 5)).all())
    assert torch.equal(dz, want[0]) and torch.equal(dzt, want[1]) and torch.equal(db, want[2])


class Insists:
    """Stands in for the native module and takes no call that it declines."""

    def __init__(self, host):
        self.host, self.taken = host, set()

    def __getattr__(self, name):
        def call(*a):
            got = getattr(self.host, name)(*a)
            assert got is not None, name
            self.taken.add(name)
            return got
        return call


def test_the_calls_are_taken_natively(monkeypatch):
    host = Insists(sp24._load_host())
    monkeypatch.setattr(sp24, "_host", host)
    for call in calls():
        call()
    assert host.taken >= {"sp24_moe_route", "sp24_moe_route_backward", "sp24_checkpoint_rows", "sp24_restore_rows", "sp24_linear_backward_checkpoint",
                          "sp24_gemm_dense_checkpoint", "sp24_gemm_dense_grouped_checkpoint", "sp24_moe_sort"}
