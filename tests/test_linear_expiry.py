"""What a walk of linear attention leaves behind when one of its waits has expired: NaN wherever it was to write, and nothing of it elsewhere.  The
kernel's own source on the host, as in test_linear_protocol.py; no GPU."""
import subprocess

import pytest

import test_cta_protocol as cp
import test_linear_protocol as lp

ONE = r"""
// places of their own for what a CTA writes; a warp stands for its first thread, so every 32nd word of an output is looked at
static const size_t kOutAt = 1 << 18, kStateAt = 1 << 20, kEndsAt = 1 << 21;
static bool spoilt(const float* at, size_t words, size_t step = 32) {
    for (size_t i = 0; i < words; i += step) if (at[i] == at[i]) return false;
    return true;
}
static bool untouched(size_t from, size_t to) {
    for (size_t i = from; i < to; ++i) if (F[i] != 0.f) return false;
    return true;
}
static std::string one(const std::string& name, const emu::Scenario& s, int i) {
    std::fill(F.begin(), F.end(), 0.f);
    const int H = 3, segments = 2, head = 1, T = 2 * 256 - (i % 3) * 40;
    LinearP p{};
    p.T = T; p.H = H; p.BH = H; p.segments = segments; p.length = 256; p.g = f() + 1024; p.scale = 1.f; p.status = u(); p.walks = 1;
    for (int h = 0; h < H; ++h) F[1024 + h] = i & 16 ? -1.f : -0.01f;
    LinearWalk& w = p.w[0];
    w.a = w.b = w.c = f(); w.reverse = i & 1; w.flip = i >> 1 & 1; w.exact = i >> 2 & 1;
    const bool ends = name == "ends";
    const int segment = ends ? (w.reverse ? 1 : 0) : i >> 3 & 1, DB = 128, DC = 64;
    w.out = ends ? nullptr : (void*)(f() + kOutAt); w.sT = ends ? nullptr : f() + kStateAt; w.ends = ends ? f() + kEndsAt : nullptr;
    LinearMaps m{};
    m.a[0] = m.b[0] = m.c[0] = box(128 * 64 * 2); m.out[0] = box(0);
    const dim3 block(head * segments + segment);
    const std::string e = ends ? emu::run(s, kTcThreads, block, dim3(1), [&] { k_linear_tc<128, 64, true>(m, p); })
                               : emu::run(s, kTcThreads, block, dim3(1), [&] { k_linear_tc<128, 64, false>(m, p); });
    if (!e.empty()) return e;
    const size_t state = DB * DC;
    if (ends) {
        const size_t at = kEndsAt + (head * segments + segment) * state;
        if (!untouched(kOutAt, kEndsAt) || !untouched(kEndsAt, at) || !untouched(at + state, F.size())) return "writes beside its sums";
        if (emu::c_expired && !spoilt(&F[at], state)) return "leaves sums";
        return emu::c_expired == (F[at] != F[at]) ? "" : "sums of a clean run are spoilt";
    }
    const int first = segment * 256, end = std::min(T, first + 256);
    const bool last = segment == (w.reverse ? 0 : 1);
    for (int t = 0; t < T; ++t)
        for (int h = 0; h < H; ++h) {
            const size_t at = kOutAt + ((size_t)t * H + h) * DC / 2;
            const bool mine = h == head && t >= first && t < end;
            if (mine && emu::c_expired ? !spoilt(&F[at], DC / 2) : !untouched(at, at + DC / 2)) return "row " + std::to_string(t);
        }
    const size_t at = kStateAt + head * state;
    if (!untouched(kOutAt + (size_t)T * H * DC / 2, at) || !untouched(at + state, F.size())) return "writes beside its outputs";
    if (!last && !untouched(at, at + state)) return "writes another segment's state";
    if (last && emu::c_expired && !spoilt(&F[at], state)) return "leaves a state";
    if (!emu::c_expired && F[0] != 0.f) return "status of a clean run";
    return "";
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("expiry")
    cpp, exe = str(d / "cta.cpp"), str(d / "cta")
    with open(cpp, "w") as fh:
        fh.write(lp._source() + cp.MAIN % ONE)
    r = subprocess.run(["g++", "-O1", "-std=c++17", "-w", "-Wno-psabi", "-I", cp.HERE, "-I", cp.CSRC, "-I", "/usr/local/cuda/include", cpp, "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[:4000]
    return exe


@pytest.mark.parametrize("kernel", ["walk", "ends"])
@pytest.mark.parametrize("expire,lose", [(0, 0), (0.0005, 0), (0.05, 0), (0.005, 0.02)], ids=["none", "rare", "early", "lost load"])
def test_a_walk_that_gave_up_leaves_no_result(program, kernel, expire, lose):
    cp._run(program, kernel, 60, expire, lose)
