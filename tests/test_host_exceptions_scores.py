"""No C++ exception leaves an entry of the delta rule, the scores or the distillation loss: a program whose allocations on the host fail calls each of them.
It says that there is a device 0 where the library asks (no GPU needed; where there is none the runtime refuses to launch)."""
import os
import subprocess

import pytest

from paper_1901_10997_amd import binding as B

ENTRIES = ["delta_step", "delta_walk", "delta_backward", "logprobs", "logprobs_top", "logprobs_backward", "distill", "distill_backward"]
SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include <new>
#include "lstm355.h"
static bool fails = false;
void* operator new(size_t n)
{
    void* const p = fails ? nullptr : std::malloc(n ? n : 1);
    if (!p) throw std::bad_alloc();
    return p;
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }
extern "C" int hipGetDevice(int* d) { *d = 0; return 0; }
extern "C" int hipFuncSetAttribute(const void*, int, int) { return 0; }
int main(int, char** argv)
{
    char* const p = (char*)0x10000;     // an address that nothing follows
    int rc = 1;
    void* const q = nullptr;
    float* const f = (float*)p;
    int* const i = (int*)p;
    const size_t big = (size_t)1 << 34;
    fails = true;
    try {
        switch (argv[1][0]) {
        case '0': rc = lstm_delta_forward(1, 2, 4, 2, 8, 8, LSTM_F32, p, 32, 16, p, 32, 16, p, 64, 32, f, 8, 4, f, 8, 4, nullptr, 1.f, f, p, 64, 32, f, nullptr, p, big, q); break;
        case '1': rc = lstm_delta_forward(99, 2, 4, 2, 8, 8, LSTM_BF16, p, 32, 16, p, 32, 16, p, 64, 32, f, 8, 4, f, 8, 4, nullptr, 1.f, f, p, 64, 32, f, f, p, big, q); break;
        case '2': rc = lstm_delta_backward(99, 2, 4, 2, 8, 8, LSTM_F32, p, 32, 16, p, 32, 16, p, 64, 32, f, 8, 4, f, 8, 4, nullptr, 1.f, f, p, 64, 32, f, p, 32, 16, p, 32, 16,
                                           p, 64, 32, f, 8, 4, f, 8, 4, f, p, big, q); break;
        case '3': rc = lstm_logprobs_forward(3, 50, LSTM_F32, p, 50, nullptr, 0, i, f, i, f, f, 0, nullptr, nullptr, p, big, q); break;
        case '4': rc = lstm_logprobs_forward(1, 100000, LSTM_BF16, p, 100000, nullptr, 0, i, f, i, f, f, 64, i, f, p, big, q); break;
        case '5': rc = lstm_logprobs_backward(3, 50, LSTM_F32, p, 50, nullptr, 0, i, f, f, nullptr, p, 50, q); break;
        case '6': rc = lstm_distill_forward(3, 50, 4, LSTM_F32, p, 50, i, 4, f, 4, nullptr, 1.f, f, f, p, big, q); break;
        case '7': rc = lstm_distill_backward(3, 50, 4, LSTM_F32, p, 50, i, 4, f, 4, nullptr, 1.f, f, f, p, 50, q); break;
        }
    } catch (...) {
        rc = 77;
    }
    fails = false;
    std::printf("%d\n", rc);
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    B.load()
    at = tmp_path_factory.mktemp("host")
    (at / "main.cpp").write_text(SOURCE)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(root, "include"), str(at / "main.cpp"), "-o", str(at / "main"), "-rdynamic", B.LIB_PATH,
                    "-Wl,-rpath," + os.path.dirname(B.LIB_PATH), "-Wl,--allow-shlib-undefined"], check=True)
    return str(at / "main")


@pytest.mark.parametrize("entry", ENTRIES)
def test_failing_allocation_is_an_error_code(program, entry):
    r = subprocess.run([program, str(ENTRIES.index(entry))], capture_output=True, text=True, timeout=120, env=dict(os.environ, HIP_VISIBLE_DEVICES="-1"))
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)
    # those with dynamic LDS come to the library's own table first, the others to the runtime, which may have an error of its own
    assert int(r.stdout) in (B.LSTM_ERR_NOMEM, B.LSTM_ERR_LAUNCH), r.stdout
