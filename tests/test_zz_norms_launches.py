"""Launches of the norms and of the conversions to and from 4 bits: no extent of a grid has 2^32 threads, of which the runtime would run a part.  The host code is compiled here from the library's sources."""
import ctypes

import pytest

import paper_2006_05664_amd as P
from test_zz_experts import U, _torch, gpu
from test_zz_experts_ways import _compile, _cut, _source


class Launches:
    """What the host code launches for a size: the kernels, their grids and how many threads a workgroup has, and which workgroup a place in a grid is."""

    def __init__(self, tmp_path):
        norm, mx4 = _source("norm.hip"), _source("mx4.hip")
        self.lib = _compile(tmp_path, """
#define __device__
#define __forceinline__ inline
typedef void *hipStream_t;
struct dim3 { unsigned x, y, z; dim3(unsigned x = 1, unsigned y = 1, unsigned z = 1) : x(x), y(y), z(z) {} };
static dim3 blockIdx, gridDim;
constexpr int kThreads = 256, kPiece = 8, OPEVO_OK = 0;
struct Norm { long rows; int width, tx; };
struct Grad { long rows; int width, tx; float *dw; };
struct Rows4 { long rows; int width, tx; };
template <typename T> struct Vec { static constexpr int n = 16 / sizeof(T); };
static int id;
static int64_t asked[2][6];
static int count;
""" + _cut(norm, "constexpr int kMostLanes", ";") + _cut(norm, "enum Way", ";") + """
template <typename T, int HOLD, bool TO8, Way WAY> void norm_rows(Norm) { id = 1000 + TO8 * 100 + HOLD * 10 + WAY; }
template <typename T, int HOLD, Way WAY> void norm_grad(Grad) { id = 2000 + HOLD * 10 + WAY; }
static void norm_grad_weight(const float *, int, int, float *) { id = 3000; }
template <typename T, int HOLD> void quantize_mx4(Rows4) { id = 4000 + HOLD; }
template <typename T, int HOLD> void dequantize_mx4(Rows4) { id = 5000 + HOLD; }
template <typename... P, typename... A> int launch(const char *, void (*k)(P...), dim3 grid, dim3 block, hipStream_t, A... args)
{
    k(args...);
    const int64_t was[6] = {id, grid.x, grid.y, grid.z, block.x, 0};
    std::copy(was, was + 6, asked[count++]);
    return 0;
}
""" + _cut(_source("rows.hpp"), "// A launch has fewer than 2^32 threads").replace("inline dim3", "static dim3") + _cut(norm, "constexpr int kCols", ";") + _cut(norm, "struct Shape {", "\n}\n")
                            + _cut(norm, "template <typename T, bool TO8>\nint run_norm(") + _cut(norm, "constexpr int64_t kGroups", ";\n") + _cut(norm, "int64_t groups_of(", "}\n")
                            + _cut(norm, "template <typename T>\nint run_grad(") + _cut(mx4, "template <typename T>\nint run_quantize4(") + _cut(mx4, "template <typename T>\nint run_dequantize4(") + """
template <typename T> void ask_of(int what, long rows, int width)
{
    static float some;
    if (what == 0) run_norm<T, false>({rows, width, 0}, nullptr);
    if (what == 1) run_norm<T, true>({rows, width, 0}, nullptr);
    if (what == 2) run_grad<T>({rows, width, 0, nullptr}, &some, &some, nullptr);
    if (what == 3) run_quantize4<T>({rows, width, 0}, nullptr);
    if (what == 4) run_dequantize4<T>({rows, width, 0}, nullptr);
}
extern "C" int ask(int what, int f32, long rows, int width, int64_t *to)
{
    count = 0;
    f32 ? ask_of<float>(what, rows, width) : ask_of<short>(what, rows, width);
    std::copy(asked[0], asked[0] + 12, to);
    return count;
}
extern "C" long block_at(unsigned x, unsigned z, unsigned grid_x) { blockIdx = dim3(x, 0, z); gridDim = dim3(grid_x); return this_block(); }
""")
        self.lib.ask.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_long, ctypes.c_int, ctypes.POINTER(ctypes.c_int64)]
        self.lib.block_at.argtypes = [ctypes.c_uint] * 3
        self.lib.block_at.restype = ctypes.c_long

    def of(self, what, dtype, rows, width):
        to = (ctypes.c_int64 * 12)()
        return [tuple(to[i * 6:i * 6 + 5]) for i in range(self.lib.ask(what, int(dtype == "f32"), rows, width, to))]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_extent_of_a_launch_has_2_to_the_32_threads(dtype, tmp_path):
    launches = Launches(tmp_path)
    n = 4 if dtype == "f32" else 8
    for what in range(5):
        for rows in (1, 1000, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, (1 << 23) - 1, 1 << 23, (1 << 23) + 5, 1 << 25, (1 << 30) + 1, (1 << 31) - 1):
            for width in (1, 5, 64 * n, 64 * n + 1, 128 * n, 256 * n, 256 * n + n, 256 * n + 1, 512 * n, 2048 * n, 2048 * n + n, 20011, 1 << 24):
                for kernel, x, y, z, threads in launches.of(what, dtype, rows, width):
                    assert y == 1 and max(x * threads, z) < 1 << 32 and z < 1 << 16, (what, rows, width, kernel, x, z, threads)
                    if kernel // 1000 in (1, 4, 5):
                        # a workgroup for each row, or for as many as its lanes hold: all there, each once
                        lanes = next(t for t in (1 << i for i in range(10)) if t >= min(512 if kernel < 2000 else 256, -(-width // (n if kernel < 2000 else 8))) and (t >= 4 or kernel // 1000 != 4))
                        assert x * z >= -(-rows // (threads // lanes)) > x * (z - 1)
                        for at in range(z):
                            assert launches.lib.block_at(0, at, x) == at * x and launches.lib.block_at(x - 1, at, x) == at * x + x - 1


@gpu
@pytest.mark.parametrize("width", [2056, 2057])
def test_more_rows_than_a_grid_has_workgroups_of_512_lanes(width):
    """2^23 rows and some, each the same small number all along: the norm is 1, in 8 bits 127, 1 / rms the number's inverse."""
    torch, _ = _torch()
    rows = (1 << 23) + 5
    number = (torch.arange(rows, device="cuda") % 7 + 1).float()
    x, y = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda"), torch.full((rows, width), float("nan"), dtype=torch.bfloat16, device="cuda")
    x.copy_(number[:, None].expand(rows, width))
    inv = torch.full((rows,), float("nan"), device="cuda")
    P.opevo_norm_rows(x.data_ptr(), width, 0, 0, 0, 0.0, P.OPEVO_BF16, rows, width, 0, 0, y.data_ptr(), width, inv.data_ptr())
    torch.cuda.synchronize()
    wrong = sum(int((part != 1).sum()) for part in y.split(1 << 20))
    assert wrong == 0
    assert bool(((inv.double() * number.double() - 1).abs() <= 4 * U).all())
    del y
    q, scale = torch.full((rows, width), 77, dtype=torch.int8, device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    P.opevo_norm_rows_i8(x.data_ptr(), width, 0, 0, 0, 0.0, P.OPEVO_BF16, rows, width, 0, 0, q.data_ptr(), width, scale.data_ptr())
    torch.cuda.synchronize()
    wrong = sum(int((part != 127).sum()) for part in q.split(1 << 20))
    assert wrong == 0
    assert bool(((scale.double() * 127 - 1).abs() <= 8 * U).all())
    del x, q
    torch.cuda.empty_cache()                    # tens of GB
