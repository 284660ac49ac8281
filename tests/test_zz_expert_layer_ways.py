"""The launches of a layer of experts, from the library's own sources: parts of an activation and of h, and pairs of tiles, as they are there.  The first launch has a workgroup for every unit of rows that an
expert can have and for every inner channel; the second takes every token once; every way that a type and kind of weights can go is gone by a size of the tests."""
import ctypes

import numpy as np
import pytest

import test_zz_expert_layer as L
import test_zz_mx4_ways as W
from test_zz_experts_ways import _compile, _cut, _source

PARTS = {"bf16": 1, "f16": 2, "f32": 3}


@pytest.fixture
def ask(tmp_path):
    source = _source("expert_layer.hip")
    parts = source[source.index("template <typename T> struct Parts"):source.index("// Where value c of a row of h stands")]
    assert parts.count("struct Parts") == 3
    lib = _compile(tmp_path, """
typedef void *hipStream_t;
struct dim3 { unsigned x, y, z; dim3(unsigned x, unsigned y = 1, unsigned z = 1) : x(x), y(y), z(z) {} };
constexpr int kStep = 128;
struct Layer { int tokens, slots, experts, width, inner, groups, group_tokens, group_unit; long ld_h; };
struct Weights8 { static constexpr int SUB = 1; };
struct Weights4 { static constexpr int SUB = 2; };
typedef short bf16;
""" + _cut(source, "enum Ending", ";") + "\n" + parts + _cut(source, "template <typename T, typename Q, Ending ENDING> constexpr int kPairs", ";") + _cut(source, "int64_t row_of_h(", "}\n") + """
static int asked[11];
template <typename T, typename Q, int W, Ending E> void layer_in(Layer) { asked[0] = E; asked[8] = kPairs<T, Q, E>; asked[9] = Parts<T>::n; asked[10] = Parts<T>::h; }
template <typename T, typename Q, int W, int S, int NC, Ending E> void layer_out(Layer p) { asked[1] = E; asked[2] = S * 10 + NC; asked[3] = p.groups; asked[4] = p.group_tokens; asked[5] = p.group_unit; }
static int grids[2][3], launches;
static int launch(const char *, void (*k)(Layer), dim3 grid, dim3 block, hipStream_t, Layer p)
{
    k(p);
    const int was[3] = {(int)grid.x, (int)grid.y, (int)block.x};
    std::copy(was, was + 3, grids[launches++]);
    return 0;
}
""" + _cut(source, "template <typename T, typename Q>\nint run_layer(") + """
extern "C" void ask(int type, int i8, int tokens, int k, int experts, int width, int inner, int *to)
{
    const Layer p = {tokens, tokens * k, experts, width, inner, 0, 0, 0, row_of_h(inner)};
    launches = 0;
    if (type == 3) i8 ? run_layer<float, Weights8>(p, nullptr) : run_layer<float, Weights4>(p, nullptr);
    else if (type == 2) i8 ? run_layer<_Float16, Weights8>(p, nullptr) : run_layer<_Float16, Weights4>(p, nullptr);
    else i8 ? run_layer<bf16, Weights8>(p, nullptr) : run_layer<bf16, Weights4>(p, nullptr);
    std::copy(asked, asked + 11, to);
    std::copy(grids[0], grids[0] + 6, to + 11);
}
""")

    def of(dtype, kind, tokens, k, experts, width, inner):
        to = (ctypes.c_int * 17)()
        lib.ask(PARTS[dtype], int(kind == "i8"), tokens, k, experts, width, inner, to)
        return list(to)
    return of


def _units(counts, per):
    return sum(-(-n // per) for n in counts)


@pytest.mark.parametrize("kind", ["i8", "mx4"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_the_launches_of_a_layer(dtype, kind, ask):
    rng = np.random.default_rng(1)
    sizes = [size[:5] for size in L.SIZES + W.LAYERS] + [(512, 1, e, 40, 300) for e in (1, 2, 500, 1024)] + [(8, 64, e, 40, 300) for e in (1, 64, 1024)]
    for tokens, k, experts, width, inner in sizes:
        first, second, parts, groups, each, unit, _, _, pairs, n, h, blocks, rows, lanes, across, down, _ = ask(dtype, kind, tokens, k, experts, width, inner)
        assert n == PARTS[dtype] and h == 3
        # a workgroup for 16 channels of a pair, as far as h goes, and one for each unit, and the plan's
        assert blocks * pairs * 16 == -(-inner // 256) * 256 and lanes == 256
        most = 0
        for _ in range(20):
            ids = rng.integers(0, experts, tokens * k) if rng.random() < 0.7 else rng.integers(0, min(experts, 3), tokens * k)
            most = max(most, _units(np.bincount(ids, minlength=experts), 16 // n))
        one_each = np.zeros(experts, dtype=int)
        one_each[:min(experts, tokens * k)] = 1
        one_each[0] += tokens * k - one_each.sum()
        assert rows - 1 >= max(most, _units(one_each, 16 // n))
        cols = parts % 10 * 16 // (parts // 10)
        assert across * cols >= width > (across - 1) * cols and down == groups and (groups - 1) * each < tokens <= groups * each
        assert unit >= 1 and unit * h <= 16 // (parts // 10)


def _ways(dtype, kind, to, tokens):
    first, second, parts, groups, each, _, _, _, pairs, *_ = to
    return {("first", first, pairs), ("second", second, parts, "one group" if groups == 1 else "a token each" if each == 1 else "groups")}


@pytest.mark.parametrize("kind", ["i8", "mx4"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_every_way_of_a_layer_is_gone(dtype, kind, ask):
    there, gone = {}, set()
    for tokens in (1, 2, 3, 7, 16, 33, 64, 128, 256, 512):
        for k in (1, 2, 4, 8):
            for width in (1, 9, 20, 64, 130, 256, 270, 512, 640, 1000, 1024, 1280, 1500, 2048, 2560, 2600, 4096, 4112, 16384):
                for inner in (1, 9, 20, 64, 128, 256, 270, 512, 1000, 1024, 2048, 4096):
                    if tokens * k <= 512:
                        for way in _ways(dtype, kind, ask(dtype, kind, tokens, k, 8, width, inner), tokens):
                            there.setdefault(way, (tokens, k, width, inner))
    for tokens, k, experts, width, inner, *_ in L.SIZES + W.LAYERS:
        gone |= _ways(dtype, kind, ask(dtype, kind, tokens, k, experts, width, inner), tokens)
    assert len(there) > 12
    assert {way: size for way, size in there.items() if way not in gone} == {}
