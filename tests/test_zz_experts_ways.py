"""Every way that an expert layer's calls can take through their kernels is one that a test goes: the host code that chooses it is compiled here from the library's sources and asked for
the ways of a wide range of sizes and of the tests' own, and the sizes below are those that the other file's lists leave out."""
import ctypes
import os
import subprocess

import pytest

import test_zz_experts as E
from host_code import CLANG, ROOT

CSRC = os.path.join(ROOT, "paper_2006_05664_amd", "csrc")


def _source(name):
    return open(os.path.join(CSRC, name)).read()


def _cut(text, start, end="\n}\n"):
    at = text.index(start)
    return text[at:text.index(end, at) + len(end)]


def _compile(tmp_path, text):
    src, lib = str(tmp_path / "t.cpp"), str(tmp_path / "t.so")
    with open(src, "w") as fh:
        fh.write("#include <algorithm>\n#include <cstdint>\n" + text)
    subprocess.run([CLANG, "-std=c++17", "-O1", "-w", "-shared", "-fPIC", src, "-o", lib], check=True)
    return ctypes.CDLL(lib)


# ------------------------------------------------------------------ routing
class Ways:
    """How a size runs, for elements of which a 16-byte piece holds n: whether rows are at least a piece, whether several waves share a row, pieces a lane holds, whether a workgroup
    goes on to further tokens or slots, and whether a row is longer than its lanes hold."""

    def __init__(self, tmp_path):
        text = _source("route.hip")
        self.lib = _compile(tmp_path, "constexpr int kThreads = 256, kOwn = 64;\nstruct Route { long tokens; int k; const int *counts; int tokens_per_block; long blocks; };\n"
                            + _cut(text, "struct Lay {", "};\n") + _cut(text, "static Lay lay_out(") + _cut(text, "void deal(Route") + _cut(text, "int slots_a_workgroup(") + """
extern "C" void lay(int64_t pieces, int64_t rows, int most, int *to) { const Lay l = lay_out(pieces, rows, most); to[0] = l.tx; to[1] = l.ty; to[2] = l.hold; }
extern "C" int dealt(int64_t tokens, int k, int counted, int ty) { Route r = {(long)tokens, k, counted ? &r.k : nullptr, 0, 0}; deal(&r, ty); return r.tokens_per_block; }
extern "C" int share(int64_t blocks, int k) { return slots_a_workgroup(blocks, k); }
""")
        self.lib.lay.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
        self.lib.dealt.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int]
        self.lib.share.argtypes = [ctypes.c_int64, ctypes.c_int]

    def lay(self, pieces, rows, most):
        to = (ctypes.c_int * 3)()
        self.lib.lay(pieces, rows, most, to)
        return tuple(to)

    def of(self, tokens, k, width, n):
        pieces, wide = -(-width // n), width >= n
        tx, ty, hold = self.lay(pieces, tokens, 4)
        each = self.lib.dealt(tokens, k, int(tokens * k > 4096), ty)
        ways = {("dispatch", wide, tx > 64, hold, min(each, tokens) > ty, pieces > tx * hold), ("quantize", wide, tx > 64, hold, pieces > tx * hold)}
        tx, ty, _ = self.lay(pieces, tokens, 1)
        blocks = -(-tokens // ty)
        parts = max(1, min(-(-pieces // tx), 1024 // blocks))
        return ways | {("gradient", wide, tx > 64, self.lib.share(blocks, k) > 1, wide and width % n != 0, pieces > tx), ("combine", wide, tx > 64, parts > 1, pieces > tx * parts)}


# tokens, k, experts, width, dtype, held, extra elements between rows, shift: ways that no size of the other list goes
ROUTES = [
    (1, 1, 3, 2060, "bf16", 1.0, 0, 0), (1, 1, 2, 4100, "f16", 1.0, 0, 0), (300, 1, 7, 8192, "bf16", 0.9, 0, 0), (513, 1, 5, 2056, "f16", 0.9, 0, 0),
    (513, 1, 12, 4100, "bf16", 1.0, 0, 0), (513, 1, 64, 8200, "f16", 0.8, 0, 0), (513, 4, 9, 1030, "bf16", 0.9, 3, 1), (513, 4, 40, 2056, "f16", 1.0, 0, 0),
    (513, 4, 31, 2060, "bf16", 0.7, 1, 3), (513, 16, 33, 260, "f16", 0.9, 0, 0), (2048, 1, 8, 260, "bf16", 1.0, 4, 0), (4096, 1, 64, 520, "f16", 0.9, 0, 0),
    (4096, 1, 3, 1030, "bf16", 1.0, 0, 0), (4096, 2, 100, 520, "f16", 0.9, 8, 0), (4200, 1, 17, 1030, "f16", 0.9, 0, 0), (12000, 64, 70, 1, "bf16", 0.9, 0, 0),
    (1100, 3, 13, 1000, "f16", 0.9, 0, 0), (2100, 4, 64, 2056, "bf16", 0.95, 0, 0), (4200, 2, 16, 1030, "f16", 0.95, 0, 0),
    (1, 1, 1, 1, "f32", 1.0, 0, 0), (1, 1, 4, 260, "f32", 1.0, 0, 0), (1, 1, 4, 1030, "f32", 1.0, 0, 0), (1, 1, 9, 2056, "f32", 1.0, 0, 0), (1, 1, 2, 4100, "f32", 1.0, 0, 0),
    (65, 1, 6, 16384, "f32", 0.8, 0, 0), (513, 1, 8, 1001, "f32", 0.9, 2, 1), (513, 1, 70, 1030, "f32", 0.9, 0, 0), (513, 1, 5, 2056, "f32", 0.9, 0, 0),
    (513, 1, 12, 4100, "f32", 1.0, 0, 0), (513, 4, 9, 1001, "f32", 0.9, 0, 0), (513, 4, 31, 1030, "f32", 0.7, 1, 3), (513, 4, 40, 1032, "f32", 1.0, 0, 0),
    (513, 16, 33, 136, "f32", 0.9, 0, 0), (4096, 1, 64, 260, "f32", 0.9, 0, 0), (4096, 1, 3, 520, "f32", 1.0, 4, 0), (4096, 2, 100, 260, "f32", 0.9, 0, 0),
    (4200, 1, 17, 520, "f32", 0.9, 0, 0), (8192, 2, 65, 130, "f32", 0.95, 0, 0), (12000, 64, 70, 1, "f32", 0.9, 0, 0), (1100, 3, 13, 1000, "f32", 0.9, 0, 0),
]


@pytest.mark.parametrize("n", [8, 4])
def test_every_way_of_the_routing_is_gone(n, tmp_path):
    ways = Ways(tmp_path)
    there, gone = {}, set()
    for tokens in (1, 2, 3, 9, 40, 65, 200, 300, 513, 700, 1024, 1100, 2048, 2100, 3000, 4096, 4200, 5000, 8192, 12000, 16390, 40000):
        for k in (1, 2, 3, 4, 5, 8, 16, 64):
            for width in (1, 3, 4, 7, 8, 33, 40, 130, 136, 260, 300, 500, 512, 520, 1000, 1001, 1024, 1030, 1032, 2048, 2056, 2060, 4096, 4100, 5000, 8192, 8200, 16384, 16400, 20000, 40000):
                if tokens * k * width <= 1.3e8:
                    for way in ways.of(tokens, k, width, n):
                        there.setdefault(way, (tokens, k, width))
    for tokens, k, _, width, dtype, *_ in E.ROUTES + ROUTES:
        if (dtype == "f32") == (n == 4):
            gone |= ways.of(tokens, k, width, n)
    assert len(there) > 30
    assert {way: size for way, size in there.items() if way not in gone} == {}


@pytest.mark.gpu
@pytest.mark.parametrize("size", ROUTES, ids=str)
def test_routing(size):
    E.test_dispatch_and_its_gradient(*size)
    E.test_combine_and_its_gradients(*size)
    E.test_dispatch_in_8_bits(*size)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [s for s in ROUTES if s[0] * s[3] <= 1 << 23], ids=str)
def test_rows_in_8_bits(size):
    tokens, _, _, width, dtype, _, pad, shift = size
    E.test_rows_in_8_bits(tokens, width, pad, shift, dtype)


# ------------------------------------------------------------------ products
def _chooser(tmp_path):
    """The kernels of either table by a number of their own, and the one that is chosen for a size."""
    lib = _compile(tmp_path, """
typedef void *hipStream_t;
struct Product { const int8_t *a, *b; long lda, ldb; const int *offsets; int experts; long m; int n, k; };
template <bool DIRECT, int BM, int BN, int WM, int WN, int STAGES, int KG = 1> struct Shape { static constexpr int id = ((DIRECT * 1000 + BM) * 1000 + BN) * 100 + STAGES * 10 + KG; };
template <typename S> int run_tile(const Product &, hipStream_t) { return S::id; }
template <int MI, int NI, int W> int run_thin(const Product &, hipStream_t) { return W; }
""" + _cut(_source("matmul_i8.hip"), "struct Kernel {", "int check_operand(").replace("int check_operand(", "") + """
extern "C" int pick(long m, int n, int k, long lda, long ldb, int experts) { const int at = 0; return run_product({nullptr, nullptr, lda, ldb, experts ? &at : nullptr, experts, m, n, k}, nullptr); }
extern "C" int kernel(int direct, int i)
{
    if (direct) return i < (int)(sizeof kDirect / sizeof *kDirect) ? kDirect[i].run({}, nullptr) : -1;
    return i < (int)(sizeof kAny / sizeof *kAny) ? kAny[i].run({}, nullptr) : -1;
}
""")
    lib.pick.argtypes = [ctypes.c_long, ctypes.c_int, ctypes.c_int, ctypes.c_long, ctypes.c_long, ctypes.c_int]
    kernels = set()
    for direct in (0, 1):
        i = 0
        while lib.kernel(direct, i) >= 0:
            kernels.add((bool(direct), lib.kernel(direct, i)))
            i += 1
    return lib, kernels


# rows of each expert, rows of none, N, K, output: 128 x 128 tiles with four stages, by one slab, five and many
GROUPS = [([100, 0, 77, 300, 8, 66, 31, 50, 3], 0, 3095, 64, "f32"), ([244, 128, 1, 310, 200, 0, 127, 100], 60, 1690, 560, "bf16"), ([400, 257, 0, 640, 130], 33, 1900, 1040, "f16")]


def test_every_kernel_of_the_products_is_chosen_plain_and_by_experts(tmp_path):
    lib, kernels = _chooser(tmp_path)
    plain, grouped = set(), set()
    for M, N, K, _, pa, pb, _, shift in E.PRODUCTS:
        plain.add((K % 16 == (K + pa) % 16 == (K + pb) % 16 == shift % 16 == 0, lib.pick(M, N, K, K + pa, K + pb, 0)))
    for M, N, K, _ in E.LARGE:
        for pad in (0, 16, 3):
            plain.add((K % 16 == (K + pad) % 16 == 0, lib.pick(M, N, K, K + pad, K + pad, 0)))
    for counts, none, N, K, _, pa, pb in [g + (0, 0) for g in E.LARGE_GROUPS + GROUPS] + E.GROUPS:
        grouped.add((K % 16 == (K + pa) % 16 == (K + pb) % 16 == 0, lib.pick(sum(counts) + none, N, K, K + pa, K + pb, len(counts))))
    assert len(kernels) > 10
    assert kernels - plain == set() and kernels - grouped == set()


@pytest.mark.gpu
@pytest.mark.parametrize("counts,none,N,K,dtype", GROUPS)
def test_products_of_experts(counts, none, N, K, dtype):
    E.test_large_products_of_experts(counts, none, N, K, dtype)
