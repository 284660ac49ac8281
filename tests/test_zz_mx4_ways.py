"""Every kernel of the 4-bit products and of the layers of experts is chosen by a size of the tests: the host code that chooses is compiled here from the library's sources and asked for a wide range of
sizes and for the tests' own, and the sizes below are those that the other files' lists leave out.  Then what holds for all of these calls: rows far apart, two streams at once, errors of others."""
import ctypes

import numpy as np
import pytest

import paper_2006_05664_amd as P
import test_zz_expert_layer as L
import test_zz_mx4 as X
from test_zz_experts import CODE, Matrix, _torch, gpu
from test_zz_experts_ways import _compile, _cut, _source


# ------------------------------------------------------------------ products
def _chooser(tmp_path):
    """The kernels of the tables by numbers of their own, and the one that is chosen for a size."""
    lib = _compile(tmp_path, """
#include <cmath>
typedef void *hipStream_t;
struct Product4 { const uint8_t *a, *b, *sa, *sb; long lda, ldb, ldsa, ldsb; const int *offsets; int experts; long m; int n, k; bool odd; };
template <bool DIRECT, int BM, int BN, int WM, int WN, int STAGES, int KG = 1> struct Shape { static constexpr int id = ((DIRECT * 1000 + BM) * 1000 + BN) * 100 + STAGES * 10 + KG; };
template <int BM, int BN, int WM, int WN, int STAGES> struct LongShape { static constexpr int id = ((2000 + BM) * 1000 + BN) * 100 + STAGES * 10; };
template <typename S> int run_tile(const Product4 &, hipStream_t) { return S::id; }
template <typename S> int run_long(const Product4 &, hipStream_t) { return S::id; }
template <int W> int run_thin(const Product4 &, hipStream_t) { return W; }
""" + _cut(_source("matmul_mx4.hip"), "struct Kernel {", "int product4(").replace("int product4(", "") + """
extern "C" int pick(long m, int n, int k, long lda, long ldb, long ldsa, long ldsb, int experts)
{
    const int at = 0;
    Product4 p = {nullptr, nullptr, nullptr, nullptr, lda, ldb, ldsa, ldsb, experts ? &at : nullptr, experts, m, n, (k + 1) / 2, k % 2 != 0};
    return run_product4(p, nullptr);
}
extern "C" int kernel(int table, int i)
{
    if (table == 0) return i < (int)(sizeof kLong / sizeof *kLong) ? kLong[i].run({}, nullptr) : -1;
    if (table == 1) return i < (int)(sizeof kDirect / sizeof *kDirect) ? kDirect[i].run({}, nullptr) : -1;
    return i < (int)(sizeof kAny / sizeof *kAny) ? kAny[i].run({}, nullptr) : -1;
}
""")
    lib.pick.argtypes = [ctypes.c_long, ctypes.c_int, ctypes.c_int] + [ctypes.c_long] * 4 + [ctypes.c_int]
    kernels = set()
    for table in range(3):
        i = 0
        while lib.kernel(table, i) >= 0:
            kernels.add((table > 1 and lib.kernel(table, i) < 100, lib.kernel(table, i)))       # the kernel without tiles is in two tables
            i += 1
    return lib, kernels


def _way(lib, M, N, K, pa, pb, pf, shift, experts=0):
    half, blocks = (K + 1) // 2, (K + 31) // 32
    kernel = lib.pick(M, N, K, half + pa, half + pb, blocks + pf, blocks + pf, experts)
    whole = K % 32 == 0 and (half + pa) % 16 == (half + pb) % 16 == 0 and (blocks + pf) % 4 == 0 and shift % 16 == 0
    return kernel < 100 and not whole, kernel


# rows of each expert, rows of none, N, K, output: kernels that no grouped size of the other file takes
GROUPS = [
    ([1300, 700, 2200, 1500], 30, 4090, 2048, "bf16"), ([1023, 2, 1500, 0, 1999], 3, 3500, 3200, "f32"), ([300, 500, 0, 129], 5, 1024, 1024, "f16"), ([200, 100, 61], 9, 640, 4096, "bf16"),
    ([3, 0, 5, 1], 2, 520, 1280, "f32"), ([2, 1, 0, 6], 1, 77, 333, "f16"),
    ([2600, 0, 4000, 3000, 2700, 3800], 46, 21, 256, "bf16"), ([20, 0, 31, 14, 18], 2, 3271, 1024, "f32"), ([17, 20, 14, 0, 30, 20], 1, 2739, 4096, "f16"), ([65, 130, 0, 100, 60, 30], 5, 2692, 256, "f32"),
    ([134, 200, 0, 166, 160], 10, 3274, 256, "bf16"),
    ([40, 0, 90, 62, 55, 38], 3, 2935, 1024, "bf16"), ([3000, 2000, 0, 6000], 4, 202, 256, "f16"), ([2700, 3100, 0, 5000, 2600, 2800], 6, 66, 640, "f32"),
]


PLAIN = [(2949, 3460, 2048, "f16"), (1361, 1531, 2048, "bf16"), (863, 1503, 4096, "f32")]


def test_every_kernel_of_the_products_is_chosen_plain_and_by_experts(tmp_path):
    lib, kernels = _chooser(tmp_path)
    plain, grouped = set(), set()
    for M, N, K, _, pa, pb, _, pf, shift in X.PRODUCTS:
        if shift == 0:
            plain.add(_way(lib, M, N, K, pa, pb, pf, shift))
    for M, N, K, _ in X.LARGE:
        for pad in (0, 16, 3):
            plain.add(_way(lib, M, N, K, pad, pad, -(-K // 32) * 7 % 4 if pad else 0, 0))
    for M, N, K, _ in PLAIN:
        plain.add(_way(lib, M, N, K, 0, 0, 0, 0))
    for counts, none, N, K, _, pa, pb in [g + (0, 0) for g in X.LARGE_GROUPS + GROUPS] + X.GROUPS:
        grouped.add(_way(lib, sum(counts) + none, N, K, pa, pb, 0, 0, len(counts)))
    assert len(kernels) > 14
    assert kernels - plain == set()
    assert kernels - grouped == set()


@gpu
@pytest.mark.parametrize("counts,none,N,K,dtype", GROUPS)
def test_products_of_experts(counts, none, N, K, dtype):
    X.test_products_of_experts(counts, none, N, K, dtype, 0, 0)


@gpu
@pytest.mark.parametrize("M,N,K,dtype", PLAIN)
def test_products(M, N, K, dtype):
    X.test_large_products(M, N, K, dtype, 0)


# ------------------------------------------------------------------ layers
class Layers:
    """How a layer runs: the kernels of both launches, and whether the second one's tokens are in groups."""

    def __init__(self, tmp_path):
        self.lib = _compile(tmp_path, """
typedef void *hipStream_t;
struct dim3 { unsigned x, y, z; dim3(unsigned x, unsigned y = 1, unsigned z = 1) : x(x), y(y), z(z) {} };
enum Ending { kEven, kRagged, kTiny };
constexpr int kStep = 128;
struct Layer { int tokens, slots, experts, width, inner, groups, group_tokens, group_unit; long ld_h; };
template <typename T> struct Parts { static constexpr int n = sizeof(T) == 4 ? 3 : 1, h = sizeof(T) == 4 ? 3 : 2; };
struct Weights8 { static constexpr int SUB = 1; };
struct Weights4 { static constexpr int SUB = 2; };
template <typename T, typename Q, Ending E> constexpr int kPairs = 2;
static int asked[8];
template <typename T, typename Q, int W, Ending E> void layer_in(Layer) { asked[0] = E; }
template <typename T, typename Q, int W, int S, int NC, Ending E> void layer_out(Layer p) { asked[1] = E; asked[2] = S * 10 + NC; asked[3] = p.groups; asked[4] = p.group_tokens; asked[5] = p.group_unit; }
static int launch(const char *, void (*k)(Layer), dim3 grid, dim3, hipStream_t, Layer p) { k(p); asked[6] = asked[7]; asked[7] = grid.y; return 0; }
""" + _cut(_source("expert_layer.hip"), "template <typename T, typename Q>\nint run_layer(") + """
extern "C" void ask(int f32, int i8, int tokens, int k, int experts, int width, int inner, int *to)
{
    const Layer p = {tokens, tokens * k, experts, width, inner, 0, 0, 0, (inner + 255L) / 256 * 256};
    if (f32) i8 ? run_layer<float, Weights8>(p, nullptr) : run_layer<float, Weights4>(p, nullptr);
    else i8 ? run_layer<short, Weights8>(p, nullptr) : run_layer<short, Weights4>(p, nullptr);
    std::copy(asked, asked + 8, to);
}
""")

    def of(self, dtype, kind, tokens, k, experts, width, inner):
        to = (ctypes.c_int * 8)()
        self.lib.ask(int(dtype == "f32"), int(kind == "i8"), tokens, k, experts, width, inner, to)
        first, second, parts, groups, each, unit, units, grid = to
        assert grid == groups and (groups - 1) * each < tokens <= groups * each and 1 <= unit * (3 if dtype == "f32" else 2) <= 16 // (parts // 10)
        return {("first", first), ("second", second, parts, "one group" if groups == 1 else "a token each" if each == 1 else "groups")}


# tokens, k, experts, width, inner, held, extra between rows, shift: ways that no size of the other list goes
LAYERS = [
    (3, 2, 4, 2064, 300, 1.0, 0, 0), (100, 2, 6, 2064, 1001, 0.9, 0, 0), (60, 3, 7, 4112, 512, 1.0, 0, 0), (200, 2, 5, 3000, 270, 0.9, 0, 0), (200, 1, 3, 4112, 12, 1.0, 0, 0), (9, 2, 3, 4112, 20, 1.0, 0, 0),
    (120, 4, 9, 640, 1024, 0.9, 0, 0), (300, 1, 9, 1500, 512, 0.9, 0, 0), (2, 2, 3, 2560, 1024, 1.0, 0, 0), (90, 1, 2, 200, 10, 1.0, 0, 0), (1, 3, 3, 4200, 9, 1.0, 0, 0), (5, 1, 2, 40, 14, 1.0, 0, 0),
    (1, 2, 3, 4112, 512, 1.0, 0, 0), (1, 2, 3, 4112, 270, 1.0, 0, 0), (30, 2, 3, 270, 12, 1.0, 0, 0), (70, 2, 3, 2560, 2048, 1.0, 0, 0), (1, 2, 3, 2560, 2048, 1.0, 0, 0), (20, 3, 4, 128, 512, 0.9, 0, 0),
    (50, 2, 4, 1100, 128, 0.9, 0, 0), (50, 2, 4, 1100, 256, 1.0, 5, 1), (40, 2, 4, 4112, 100, 0.9, 0, 0), (60, 2, 3, 1030, 9, 1.0, 1, 3),
    (20, 2, 4, 130, 1024, 1.0, 0, 0), (17, 2, 4, 72, 512, 0.9, 0, 0), (5, 2, 4, 130, 1024, 1.0, 0, 0), (5, 2, 4, 130, 512, 1.0, 3, 1),
]


@pytest.mark.parametrize("kind", ["i8", "mx4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_way_of_a_layer_is_gone(dtype, kind, tmp_path):
    ways = Layers(tmp_path)
    there, gone = {}, set()
    for tokens in (1, 2, 3, 7, 16, 33, 64, 100, 128, 200, 256, 512):
        for k in (1, 2, 3, 4, 8):
            for width in (1, 9, 15, 20, 30, 64, 128, 200, 256, 270, 512, 640, 1000, 1024, 1280, 1500, 2048, 2560, 2600, 3584, 4096, 4112, 8192, 16384):
                for inner in (1, 9, 15, 20, 30, 64, 128, 256, 270, 512, 768, 1000, 1024, 1536, 2048, 4096):
                    if tokens * k <= 512:
                        for way in ways.of(dtype, kind, tokens, k, 8, width, inner):
                            there.setdefault(way, (tokens, k, width, inner))
    for tokens, k, experts, width, inner, *_ in L.SIZES + LAYERS:
        gone |= ways.of(dtype, kind, tokens, k, experts, width, inner)
    assert len(there) > 12
    assert {way: size for way, size in there.items() if way not in gone} == {}


@gpu
@pytest.mark.parametrize("kind", ["i8", "mx4"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", LAYERS, ids=str)
def test_layers(size, dtype, kind):
    L.test_layers(*size, dtype, kind)


# ------------------------------------------------------------------ all of them
@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_more_than_32_bits_apart(dtype):
    """Three rows over 2^31 elements from end to end: quantisation and back, and products whose operands stand like that."""
    torch, types = _torch()
    far, width, half, blocks = (1 << 30) + 64, 96, 48, 3
    g = torch.Generator(device="cuda").manual_seed(4)
    buf = torch.empty(2 * far + width, dtype=types[dtype], device="cuda")
    x = torch.as_strided(buf, (3, width), (far, 1))
    x.copy_(torch.randn(3, width, generator=g, device="cuda"))
    small = x.contiguous()
    qs, bs = torch.empty(3, half, dtype=torch.uint8, device="cuda"), torch.empty(3, blocks, dtype=torch.uint8, device="cuda")
    P.opevo_quantize_rows_mx4(small.data_ptr(), width, CODE[dtype], 3, width, qs.data_ptr(), half, bs.data_ptr(), blocks)
    qbuf, bbuf = (torch.empty(2 * far + half, dtype=torch.uint8, device="cuda") for _ in range(2))
    q, b = torch.as_strided(qbuf, (3, half), (far, 1)), torch.as_strided(bbuf, (3, blocks), (far, 1))
    P.opevo_quantize_rows_mx4(buf.data_ptr(), far, CODE[dtype], 3, width, qbuf.data_ptr(), far, bbuf.data_ptr(), far)
    torch.cuda.synchronize()
    assert torch.equal(q, qs) and torch.equal(b, bs)
    want = torch.empty_like(small)
    P.opevo_dequantize_rows_mx4(qs.data_ptr(), half, bs.data_ptr(), blocks, CODE[dtype], 3, width, want.data_ptr(), width)
    x.fill_(7.0)
    P.opevo_dequantize_rows_mx4(qbuf.data_ptr(), far, bbuf.data_ptr(), far, CODE[dtype], 3, width, buf.data_ptr(), far)
    torch.cuda.synchronize()
    assert torch.equal(x, want)
    c, cs = torch.empty(3, 3, device="cuda"), torch.empty(3, 3, device="cuda")
    P.opevo_matmul_mx4(qbuf.data_ptr(), far, bbuf.data_ptr(), far, qbuf.data_ptr(), far, bbuf.data_ptr(), far, c.data_ptr(), 3, P.OPEVO_F32, 3, 3, width)
    v = want.double()
    torch.cuda.synchronize()
    cs = torch.matmul(v, v.t().contiguous())
    # bf16 holds the values of codes exactly: a code has two bits
    assert bool(((c.double() - cs).abs() <= 2.0 ** -24 * 4 * 9 * torch.matmul(v.abs(), v.abs().t().contiguous())).all())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_layer_on_two_streams_at_once(dtype):
    """Calls on two streams with a workspace each, many times over: each one's result is what it is alone."""
    torch, types = _torch()
    g = torch.Generator(device="cuda").manual_seed(8)
    tokens, k, experts, width, inner = 40, 3, 11, 500, 260
    win, wout = L.Weights(g, experts * 2 * inner, width, "mx4"), L.Weights(g, experts * width, inner, "mx4")
    size = P.opevo_expert_layer_workspace(tokens, k, CODE[dtype], inner)
    sides = []
    for _ in range(2):
        x = Matrix(tokens, width, dtype, values=torch.randn(tokens, width, generator=g, device="cuda").cpu().numpy())
        ids = torch.randint(0, experts, (tokens, k), generator=g, device="cuda", dtype=torch.int32)
        y, ws = Matrix(tokens, width, dtype), torch.empty(size, dtype=torch.uint8, device="cuda")
        L._call("mx4", x, dtype, ids, None, tokens, k, experts, width, inner, win, wout, y, ws, size)
        sides.append((x, ids, y, ws, y.host().copy(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _, _, y, ws, _, _ in sides:
        y.view.zero_()
        ws.fill_(255)
    torch.cuda.synchronize()
    for _ in range(20):
        for x, ids, y, ws, _, stream in sides:
            L._call("mx4", x, dtype, ids, None, tokens, k, experts, width, inner, win, wout, y, ws, size, stream.cuda_stream)
    torch.cuda.synchronize()
    for _, _, y, _, alone, _ in sides:
        assert np.array_equal(y.host(), alone)


@gpu
def test_an_error_of_another_call_is_not_this_one_s():
    torch, _ = _torch()
    hip = P.binding.lib                         # the runtime that the library is bound to
    rows, width = 16, 64
    x, w, y, dx = torch.randn(rows, width, device="cuda"), torch.ones(width, device="cuda"), *(torch.empty(rows, width, device="cuda") for _ in range(2))
    inv, dw = torch.empty(rows, device="cuda"), torch.empty(width, device="cuda")
    q8, scale = torch.empty(rows, width, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    q, b, c = torch.empty(rows, width // 2, dtype=torch.uint8, device="cuda"), torch.empty(rows, 2, dtype=torch.uint8, device="cuda"), torch.empty(rows, rows, device="cuda")
    offsets, ids = torch.tensor([0, rows], dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    w8, s8, w4, b4 = (torch.ones(2 * width * width, dtype=t, device="cuda") for t in (torch.int8, torch.float32, torch.uint8, torch.uint8))
    f32 = P.OPEVO_F32
    grad, layer = P.opevo_norm_rows_grad_workspace(rows, width), P.opevo_expert_layer_workspace(rows, 1, f32, width)
    ws = torch.empty(max(grad, layer), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    tokens = (x.data_ptr(), width, f32, ids.data_ptr(), 0, rows, 1, 1, width, width)
    calls = [
        (P.opevo_norm_rows, x.data_ptr(), width, 0, 0, w.data_ptr(), 1e-6, f32, rows, width, 0, 0, y.data_ptr(), width, inv.data_ptr()),
        (P.opevo_norm_rows_i8, x.data_ptr(), width, 0, 0, w.data_ptr(), 1e-6, f32, rows, width, 0, 0, q8.data_ptr(), width, scale.data_ptr()),
        (P.opevo_norm_rows_grad, y.data_ptr(), width, 0, 0, x.data_ptr(), width, w.data_ptr(), inv.data_ptr(), f32, rows, width, dx.data_ptr(), width, dw.data_ptr(), ws.data_ptr(), grad),
        (P.opevo_quantize_rows_mx4, x.data_ptr(), width, f32, rows, width, q.data_ptr(), width // 2, b.data_ptr(), 2),
        (P.opevo_dequantize_rows_mx4, q.data_ptr(), width // 2, b.data_ptr(), 2, f32, rows, width, y.data_ptr(), width),
        (P.opevo_matmul_mx4, q.data_ptr(), width // 2, b.data_ptr(), 2, q.data_ptr(), width // 2, b.data_ptr(), 2, c.data_ptr(), rows, f32, rows, rows, width),
        (P.opevo_matmul_mx4_grouped, q.data_ptr(), width // 2, b.data_ptr(), 2, q.data_ptr(), width // 2, b.data_ptr(), 2, offsets.data_ptr(), 1, c.data_ptr(), rows, f32, rows, rows, width),
        (P.opevo_expert_layer_i8, *tokens, w8.data_ptr(), width, s8.data_ptr(), w8.data_ptr(), width, s8.data_ptr(), y.data_ptr(), width, ws.data_ptr(), layer),
        (P.opevo_expert_layer_mx4, *tokens, w4.data_ptr(), width // 2, b4.data_ptr(), 2, w4.data_ptr(), width // 2, b4.data_ptr(), 2, y.data_ptr(), width, ws.data_ptr(), layer),
    ]
    failed = []
    for call, *args in calls:
        assert hip.hipSetDevice(1 << 20) == 101                     # refused by the runtime, which keeps the error for who asks next
        try:
            call(*args)
        except P.OpevoError as e:
            failed.append((call.__name__, str(e)))
        finally:
            left = hip.hipGetLastError()
        if left != 101:
            failed.append((call.__name__, "took the error away", left))
    assert hip.hipGetLastError() == 0
    torch.cuda.synchronize()
    assert failed == []


@gpu
@pytest.mark.parametrize("kind", ["i8", "mx4"])
def test_the_longest_inner_rows_of_the_most_slots(kind):
    """Rows of the layer's workspace beyond 2^31 bytes: 512 slots of 2^20 inner channels in three parts are 3 * 2^30."""
    torch, _ = _torch()
    tokens, width, inner, g = 512, 2, 1 << 20, torch.Generator(device="cuda").manual_seed(3)
    win, wout = L.Weights(g, 2 * inner, width, kind), L.Weights(g, width, inner, kind)
    xv = torch.randn(tokens, width, generator=g, device="cuda").cpu().numpy()
    x, y = Matrix(tokens, width, "f32", values=xv), Matrix(tokens, width, "f32")
    ids = np.zeros((tokens, 1), dtype=np.int32)
    d_ids = torch.zeros(tokens, dtype=torch.int32, device="cuda")
    size = P.opevo_expert_layer_workspace(tokens, 1, P.OPEVO_F32, inner)
    assert size > 3 << 30
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    L._call(kind, x, "f32", d_ids, None, tokens, 1, 1, width, inner, win, wout, y, ws, size)
    got, some = y.host(), np.array([0, 1, 200, 341, 342, 510, 511])
    L._layer.dtype = "f32"
    want, err = (v.cpu().numpy() for v in L._layer(x.view.double()[torch.from_numpy(some).cuda()], ids[some], None, win, wout, 1, inner))
    assert np.all(np.abs(got[some] - want) <= err + 2.0 ** -24 * np.abs(want) * 1.001 + 2.0 ** -149)
