"""What the warps of the linear attention walk tell each other, in any order of the warps and with waits that expire: the kernel's own source on
the host, as in test_cta_protocol.py.  No GPU."""
import os
import re
import subprocess

import pytest

import test_cta_protocol as cp

ONE = r"""
static std::string one(const std::string& name, const emu::Scenario& s, int i) {
    const int chunks = 1 + i % 7;
    LinearP p{};
    p.T = 128 * chunks - (i % 3) * 40; p.H = 1; p.BH = 1; p.segments = 1; p.length = 128 * chunks; p.g = f() + 1024; F[1024] = i & 16 ? -1.f : -0.01f; p.scale = 1.f; p.status = u(); p.walks = 1;
    LinearWalk& w = p.w[0];
    w.a = w.b = w.c = f(); w.out = h(); w.sT = f(); w.ends = f(); w.reverse = i & 1; w.flip = i >> 1 & 1; w.exact = i >> 2 & 1;
    auto go = [&](auto kern, int db, int dc) {
        LinearMaps m{};
        m.a[0] = m.b[0] = box(128 * 64 * 2); m.c[0] = box(128 * 64 * 2); m.out[0] = box(0);
        return emu::run(s, kTcThreads, dim3(0), dim3(1), [&] { kern(m, p); });
    };
    if (name == "ends") {
        p.segments = 2; p.length = 128 * chunks; p.T = 256 * chunks; w.out = nullptr; w.reverse = 0;
        return i & 1 ? go(k_linear_tc<128, 64, true>, 128, 64) : go(k_linear_tc<64, 128, true>, 64, 128);
    }
    switch (i & 3) {
        case 0: return go(k_linear_tc<128, 128, false>, 128, 128);
        case 1: return go(k_linear_tc<64, 64, false>, 64, 64);
        case 2: return go(k_linear_tc<64, 128, false>, 64, 128);
        default: return go(k_linear_tc<128, 64, false>, 128, 64);
    }
}
"""


# the packed arithmetic that the kernel takes from rows.cuh
ROWS = """
namespace qd { typedef unsigned long long f2; inline f2 pack2(float, float) { return 0; } inline float2 unpack2(f2) { return {0.f, 0.f}; }
inline f2 mul2(f2, f2) { return 0; } inline f2 fma2(f2, f2, f2) { return 0; } inline f2 both(float) { return 0; } inline f2 add2(f2, f2) { return 0; } }
namespace qd { inline void see_unfit(uint32_t& seen, uint32_t, uint32_t) { seen |= emu::c->rng() % 4 == 0; } inline bool seen_unfit(uint32_t seen) { return seen; } }
template <int N> void give_registers() {} template <int N> void take_registers() {}
inline int atomicMin(int* p, int x) { const int o = *p; *p = std::min(o, x); return o; }
inline float __int_as_float(int x) { return (float)x; }
inline unsigned __byte_perm(unsigned, unsigned, unsigned) { return 0; }
"""


def _source():
    read = lambda n: open(os.path.join(cp.CSRC, n)).read()  # noqa: E731
    src = read("linear_tc.cu")
    src = src[:src.index("\ntemplate <int DB, int DC, bool ENDS>\ncudaError_t launch")] + "\n}\n}\n"
    head = re.sub(r'#include "sm100\.cuh"|#pragma once', "", read("linear.cuh"))
    src = src.replace('#include "rows.cuh"', ROWS).replace('#include "linear.cuh"', head).replace("extern __shared__ unsigned char smem_raw[];", "unsigned char* const smem_raw = emu::smem;")
    src = src.replace("__shared__ ", "static ").replace("__grid_constant__ ", "").replace("__noinline__ ", "")
    src = re.sub(r"__launch_bounds__\([^)]*\)", "", src)
    assert "asm " not in src
    return '#include "cta_emulation.h"\ntypedef __nv_bfloat16 bf16;\n' + src


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("emu")
    cpp, exe = str(d / "cta.cpp"), str(d / "cta")
    with open(cpp, "w") as fh:
        fh.write(_source() + cp.MAIN % ONE)
    r = subprocess.run(["g++", "-O1", "-std=c++17", "-w", "-Wno-psabi", "-I", cp.HERE, "-I", cp.CSRC, "-I", "/usr/local/cuda/include", cpp, "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[:4000]
    return exe


@pytest.mark.parametrize("kernel", ["walk", "ends"])
def test_any_order_of_warps(program, kernel):
    cp._run(program, kernel, 200, 0, 0)


@pytest.mark.parametrize("kernel", ["walk", "ends"])
@pytest.mark.parametrize("expire,lose", [(0.0005, 0), (0.05, 0), (0.005, 0.02)], ids=["rare", "early", "lost load"])
def test_expired_waits(program, kernel, expire, lose):
    cp._run(program, kernel, 200, expire, lose)


def test_registers_that_the_state_takes(tmp_path):
    """setmaxnreg.inc waits until the CTA's own registers, those of its launch, have room: what the compiler launches has to be what the shares
    were made from."""
    from paper_2606_08804_b200 import build
    build.build()
    log = os.path.join(build.OBJ_DIR, "linear_tc.log")
    if not os.path.exists(log):
        pytest.skip("the library was not built here")
    src = open(os.path.join(cp.CSRC, "linear_tc.cu")).read()
    launch, group, state = map(int, re.search(r"kLaunchRegs = (\d+), kGroupRegs = (\d+), kStateRegs = (\d+)", src).groups())
    regs = re.findall(r"Compiling entry function '\w*k_linear_tc\w*' for 'sm_100a'(?:(?!Compiling entry).)*?Used (\d+) registers", open(log).read(), re.S)
    assert len(regs) == 8 and set(map(int, regs)) == {launch} and group + state <= 2 * launch
    assert all(r % 8 == 0 and 24 <= r <= 256 for r in (launch, group, state))
