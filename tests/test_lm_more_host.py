"""CPU checks of layer norm, distillation and sampling (include/mv_lm.h): the refusals that happen before anything is enqueued."""
import ctypes
import math
import os
import subprocess

import pytest

from paper_2011_06495_b200 import binding as B
from paper_2011_06495_b200 import build as BUILD


@pytest.fixture(scope="module")
def lib():
    BUILD.build()
    return B.load()


at = ctypes.c_void_p
P, Q, R, S, ODD = at(0x100000), at(0x200000), at(0x300000), at(0x400000), at(0x100001)      # never dereferenced
BAD = B.MV_ERR_INVALID_ARG


def test_layer_norm_refusals(lib):
    ok = dict(x=P, xt=B.MV_BF16, T=4, D=8, ldx=8, w=Q, b=Q, wt=B.MV_F32, eps=1e-5, y=R, ldy=8, m=None, r=None)

    def call(**k):
        a = {**ok, **k}
        return lib.mv_layer_norm(None, a["x"], a["xt"], a["T"], a["D"], a["ldx"], a["w"], a["b"], a["wt"], a["eps"], a["y"], a["ldy"], a["m"], a["r"])

    for k in (dict(x=None), dict(xt=B.MV_I32), dict(T=-1), dict(T=1 << 31), dict(D=0), dict(D=1 << 31), dict(ldx=7), dict(wt=B.MV_F16), dict(wt=B.MV_I64), dict(eps=-1e-9),
              dict(eps=math.nan), dict(eps=math.inf), dict(y=None), dict(ldy=7), dict(x=ODD), dict(y=ODD), dict(w=at(0x200002)), dict(b=ODD), dict(m=at(0x400002)), dict(r=ODD),
              dict(y=at(0x100002)), dict(y=at(0x100000 - 2)), dict(y=P, ldy=9), dict(y=Q), dict(w=at(0x300020))):
        assert call(**k) == BAD, k
    assert call(T=0) == B.MV_OK and call(T=0, x=None, y=None) == B.MV_OK


def test_layer_norm_grad_refusals_and_workspace(lib):
    need = B.layer_norm_grad_workspace_bytes(100, 8)
    assert need >= 64 and need % 16 == 0
    assert all(B.layer_norm_grad_workspace_bytes(*a) == 0 for a in ((-1, 8), (1 << 31, 8), (4, 0), (4, 1 << 31)))
    assert B.layer_norm_grad_workspace_bytes(0, 8) > 0
    ok = dict(dy=P, lddy=8, x=Q, ldx=8, xt=B.MV_F32, T=100, D=8, w=R, wt=B.MV_F32, m=R, r=R, dx=S, lddx=8, dw=at(0x500000), db=at(0x500020), acc=0, ws=R, n=need)

    def call(**k):
        a = {**ok, **k}
        return lib.mv_layer_norm_grad(None, a["dy"], a["lddy"], a["x"], a["ldx"], a["xt"], a["T"], a["D"], a["w"], a["wt"], a["m"], a["r"], a["dx"], a["lddx"], a["dw"], a["db"],
                                      a["acc"], a["ws"], a["n"])

    for k in (dict(dy=None), dict(x=None), dict(lddy=7), dict(ldx=7), dict(lddx=7), dict(xt=9), dict(T=-1), dict(D=0), dict(wt=B.MV_BF16), dict(m=None), dict(r=None), dict(m=ODD),
              dict(dx=None, dw=None, db=None), dict(acc=2), dict(ws=at(0x300008)), dict(dw=ODD), dict(db=at(0x500022)), dict(dx=ODD), dict(dx=at(0x100020)), dict(dx=P, lddx=9),
              dict(dx=at(0x200004)), dict(dw=P), dict(dw=Q), dict(dw=S), dict(db=at(0x300010)), dict(db=at(0x500010)), dict(w=at(0x400000))):
        assert call(**k) == BAD, k
    assert call(ws=None) == B.MV_ERR_WORKSPACE and call(n=need - 1) == B.MV_ERR_WORKSPACE


def test_distill_refusals(lib):
    ok = dict(x=P, xt=B.MV_BF16, T=4, V=30, ld=30, a=Q, i=R, it=B.MV_I64, k=3, rest=1, c=1.0, kl=S, lse=None, lr=None)

    def call(**k):
        a = {**ok, **k}
        return lib.mv_distill(None, a["x"], a["xt"], a["T"], a["V"], a["ld"], a["a"], a["i"], a["it"], a["k"], a["rest"], a["c"], a["kl"], a["lse"], a["lr"])

    for k in (dict(x=None), dict(xt=B.MV_I32), dict(T=-1), dict(T=1 << 31), dict(V=0), dict(V=1 << 31), dict(ld=29), dict(a=None), dict(i=None), dict(it=B.MV_F32), dict(k=0),
              dict(k=B.MV_TEACHER_MAX + 1), dict(rest=2), dict(rest=0, lr=S), dict(c=0.0), dict(c=-1.0), dict(c=math.nan), dict(c=math.inf), dict(x=ODD), dict(a=at(0x200002)),
              dict(i=at(0x300004)), dict(kl=ODD), dict(lse=ODD), dict(lr=ODD)):
        assert call(**k) == BAD, k
    assert call(T=0) == B.MV_OK and call(T=0, x=None, a=None, i=None) == B.MV_OK


def test_distill_grad_refusals(lib):
    ok = dict(x=P, xt=B.MV_F32, T=4, V=30, ld=30, a=Q, i=R, it=B.MV_I32, k=3, c=1.0, lse=S, lr=None, g=S, dx=at(0x500000), ldg=30)

    def call(**k):
        a = {**ok, **k}
        return lib.mv_distill_grad(None, a["x"], a["xt"], a["T"], a["V"], a["ld"], a["a"], a["i"], a["it"], a["k"], a["c"], a["lse"], a["lr"], a["g"], a["dx"], a["ldg"])

    for k in (dict(x=None), dict(xt=7), dict(T=-1), dict(V=0), dict(ld=29), dict(ldg=29), dict(a=None), dict(i=None), dict(it=B.MV_F16), dict(k=0), dict(k=1025), dict(c=0.0), dict(c=math.nan),
              dict(lse=None), dict(g=None), dict(dx=None), dict(x=ODD), dict(dx=ODD), dict(lse=ODD), dict(lr=ODD), dict(g=ODD), dict(dx=at(0x100004)), dict(dx=P, ldg=31), dict(dx=Q),
              dict(dx=at(0x300000 - 4))):
        assert call(**k) == BAD, k
    assert call(T=0) == B.MV_OK


def test_sample_refusals(lib):
    ok = dict(x=P, xt=B.MV_F16, T=4, V=30, ld=30, u=Q, c=None, k=None, p=None, m=None, y=R, it=B.MV_I64, lp=None)

    def call(**k):
        a = {**ok, **k}
        return lib.mv_sample(None, a["x"], a["xt"], a["T"], a["V"], a["ld"], a["u"], a["c"], a["k"], a["p"], a["m"], a["y"], a["it"], a["lp"])

    for k in (dict(x=None), dict(xt=B.MV_I64), dict(T=-1), dict(T=1 << 31), dict(V=0), dict(V=1 << 31), dict(ld=29), dict(u=None), dict(y=None), dict(it=B.MV_BF16), dict(x=ODD), dict(u=ODD),
              dict(c=ODD), dict(k=ODD), dict(p=ODD), dict(m=ODD), dict(y=at(0x300004)), dict(lp=ODD)):
        assert call(**k) == BAD, k
    assert call(T=0) == B.MV_OK


def test_tensors_and_streams_of_another_device_than_the_current_one(monkeypatch):
    class Stream:
        def __init__(self, device):
            self.device_index, self.cuda_stream = device, 0x1234

    monkeypatch.setattr(B, "_current_device", lambda: 1)
    monkeypatch.setattr(B, "_raw_current_stream", lambda device: 0x5678)
    assert B._raw_stream(1, None) == 0x5678 and B._raw_stream(1, Stream(1)) == 0x1234
    for device, stream in ((0, None), (0, Stream(0)), (1, Stream(0))):
        with pytest.raises(B.MvError):
            B._raw_stream(device, stream)


def test_a_gradient_of_the_distillation_that_shares_bytes_with_what_its_rows_are_weighed_by(lib):
    """dlogits: 4 rows of 30 floats from 0x500000 on, 480 bytes; with a pitch of 40, gaps of 40 bytes behind each row."""
    def call(ldg=30, lse=S, lr=S, g=S):
        return lib.mv_distill_grad(None, P, B.MV_F32, 4, 30, 30, Q, R, B.MV_I32, 3, 1.0, lse, lr, g, at(0x500000), ldg)

    for where in ("lse", "lr", "g"):
        for inside in (0x500000, 0x500000 + 476, 0x500000 - 12):
            assert call(**{where: at(inside)}) == BAD, (where, inside)
        assert call(ldg=40, **{where: at(0x500000 + 108)}) == BAD and call(ldg=40, **{where: at(0x500000 + 148)}) == BAD


def test_statistics_of_the_layer_norm_that_share_bytes_with_anything(lib):
    """x: 4 rows of 8 bf16 in a pitch of 8, 64 bytes from 0x100000 on; weight and bias: 32 bytes from 0x200000 and 0x200100 on; y from 0x300000 on."""
    def call(m=S, r=at(0x500000), ldy=8, y=R):
        return lib.mv_layer_norm(None, P, B.MV_BF16, 4, 8, 8, Q, at(0x200100), B.MV_F32, 1e-5, y, ldy, m, r)

    for inside in (0x100000, 0x10003c, 0x100000 - 12, 0x200000, 0x20001c, 0x200100 - 4, 0x300000, 0x30003c):
        assert call(m=at(inside)) == BAD and call(r=at(inside)) == BAD, hex(inside)
    assert call(r=S) == BAD and call(r=at(0x400000 + 12)) == BAD
    assert call(ldy=16, m=at(0x300000 + 8)) == BAD and call(y=P, m=at(0x100020)) == BAD


def test_gradients_of_the_layer_norm_that_share_bytes_with_statistics_or_workspace(lib):
    """x, dy, dx: 100 rows of 8 floats, 3200 bytes from 0x100000, 0x200000 and 0x300000 on; vectors and the workspace behind them."""
    need = B.layer_norm_grad_workspace_bytes(100, 8)

    def call(dx=R, m=S, r=at(0x500000), dw=at(0x600000), ws=at(0x700000), w=at(0x600100)):
        return lib.mv_layer_norm_grad(None, P, 8, Q, 8, B.MV_F32, 100, 8, w, B.MV_F32, m, r, dx, 8, dw, None, 0, ws, need)

    for inside in (0x300000, 0x300c7c, 0x300000 - 396):
        assert call(m=at(inside)) == BAD and call(r=at(inside)) == BAD
    for other in (0x100000, 0x200000, 0x300000, 0x400000, 0x500000, 0x600000, 0x600100):
        for ws in (other, other - need + 16, other + 16):
            assert call(ws=at(ws)) == BAD, hex(ws)
    assert lib.mv_layer_norm_grad(None, P, 8, Q, 8, B.MV_F32, 100, 8, None, B.MV_F32, S, S, R, 8, None, at(0x700010), 0, at(0x700000), need) == BAD
    assert lib.mv_layer_norm_grad(None, P, 8, Q, 8, B.MV_F32, 100, 8, None, B.MV_F32, S, S, R, 8, at(0x700000 - 16), None, 0, at(0x700000), need) == BAD


def test_results_of_the_distillation_that_share_bytes_with_its_inputs(lib):
    """logits: 4 rows of 30 bf16, 240 bytes from 0x100000 on; alternatives and ids: 48 and 96 bytes from 0x200000 and 0x300000 on."""
    def call(kl=S, lse=at(0x500000), lr=at(0x600000)):
        return lib.mv_distill(None, P, B.MV_BF16, 4, 30, 30, Q, R, B.MV_I64, 3, 1, 1.0, kl, lse, lr)

    for name in ("kl", "lse", "lr"):
        for inside in (0x100000, 0x1000ec, 0x100000 - 12, 0x200000, 0x20002c, 0x300000, 0x30005c):
            assert call(**{name: at(inside)}) == BAD, (name, hex(inside))
    assert call(lse=S) == BAD and call(lr=S) == BAD and call(lr=at(0x500000 + 12)) == BAD


def test_tokens_and_log_probabilities_that_share_bytes_with_what_other_rows_read(lib):
    """logits: 4 rows of 30 f16, 240 bytes from 0x100000 on; u from 0x200000, settings behind it."""
    def call(y=R, it=B.MV_I64, lp=S, c=at(0x200100), k=at(0x200200), p=at(0x200300), m=at(0x200400)):
        return lib.mv_sample(None, P, B.MV_F16, 4, 30, 30, Q, c, k, p, m, y, it, lp)

    for inside in (0x100000, 0x1000e8, 0x100000 - 8):
        assert call(y=at(inside)) == BAD and call(lp=at(inside)) == BAD and call(y=at(inside), it=B.MV_I32) == BAD
    for other in (0x200000, 0x200100, 0x200200, 0x200300, 0x200400):
        assert call(y=at(other)) == BAD and call(y=at(other + 4), it=B.MV_I32) == BAD and call(lp=at(other + 12)) == BAD and call(lp=at(other - 4)) == BAD
    assert call(lp=R) == BAD and call(lp=R, it=B.MV_I32) == BAD and call(lp=at(0x300000 + 28)) == BAD


TWO_THREADS = r"""
#include <chrono>
#include <condition_variable>
#include <cstdio>
#include <mutex>
#include <thread>
#include "mv_lm.cuh"

std::mutex m;
std::condition_variable cv;
bool slow_inside = false;
int granted = 0;                     // what the driver last heard

extern "C" cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
extern "C" cudaError_t cudaGetLastError() { return cudaSuccess; }
extern "C" cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int bytes) {
  if (bytes == 50000) {
    { std::lock_guard<std::mutex> l(m); slow_inside = true; }
    cv.notify_all();
    std::this_thread::sleep_for(std::chrono::milliseconds(200));
  }
  std::lock_guard<std::mutex> l(m);
  granted = bytes;
  return cudaSuccess;
}
static char kernel;                  // stands for one

int main() {
  static SmemLimit limit;
  bool ok[2];
  std::thread small([&] { ok[0] = allow_smem(&kernel, 50000, &limit); });
  std::thread large([&] {
    { std::unique_lock<std::mutex> l(m); cv.wait(l, [] { return slow_inside; }); }
    ok[1] = allow_smem(&kernel, 60000, &limit);
  });
  small.join();
  large.join();
  std::printf("%d\n", granted);
  return ok[0] && ok[1] && granted == 60000 && allow_smem(&kernel, 55000, &limit) && granted == 60000 ? 0 : 1;
}
"""


def test_two_threads_that_ask_for_shared_memory_of_one_kernel_at_once(tmp_path):
    """The smaller request, begun first and answered last, must not take back what the larger one was granted."""
    csrc = os.path.join(os.path.dirname(BUILD.__file__), "csrc")
    cuda = os.path.dirname(os.path.dirname(BUILD.nvcc_path()))
    (tmp_path / "two.cpp").write_text(TWO_THREADS)
    exe = str(tmp_path / "two")
    subprocess.run(["g++", "-std=c++17", "-w", "-I", csrc, "-I", os.path.join(cuda, "include"), str(tmp_path / "two.cpp"), "-o", exe, "-pthread"], check=True, timeout=300)
    assert subprocess.run([exe], timeout=60, capture_output=True).returncode == 0
