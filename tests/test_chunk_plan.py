"""Host check of how attention of a chunk is cut (csrc/chunk_plan.h), as its kernels run it.

The header is compiled for the host, 64 contexts that meet at every exchange standing in for a wavefront's lanes.  For each span of a call the pieces are
walked and, where the span begins a tile and does not end it, the pieces of that tile counted, as the kernels do; then
  * the pieces of every tile, in the order of the spans, are its steps from the first to the last, nothing lost and nothing twice;
  * a tile in one piece has no partial result; one in several has them where the merge looks for them (the second place of the span that begins it, the
    first places of the spans behind that one), and as many as its record says;
  * no place is written twice, and no record is left without its tile.
"""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

SHIM = r"""
#include <setjmp.h>
#include <stdint.h>
#include <string.h>
#include <ucontext.h>
#include <vector>

// ---- a wavefront: lanes run one after the other, up to the next exchange of values
namespace lanes {
constexpr int N = 64;
static ucontext_t first[N], home;
static jmp_buf at[N];
static char stack[N][1 << 16];
static bool started[N];
static int me, uneven;
static unsigned met[N];
static uint64_t slot[2][N];
static void (*body)();
static void resume(int i)
{
    me = i;
    if (started[i]) _longjmp(at[i], 1);
    started[i] = true;
    setcontext(&first[i]);
}
static void entry()
{
    body();
    if (me == N - 1) setcontext(&home);
    resume(me + 1);
}
static void run(void (*f)())
{
    body = f;
    for (int i = 0; i < N; ++i) {
        started[i] = false;
        met[i] = 0;
        getcontext(&first[i]);
        first[i].uc_stack.ss_sp = stack[i];
        first[i].uc_stack.ss_size = sizeof stack[i];
        makecontext(&first[i], entry, 0);
    }
    volatile bool begun = false;
    getcontext(&home);
    if (!begun) {
        begun = true;
        resume(0);
    }
}
// what every lane has: good until the next exchange
template <typename T>
const uint64_t *exchange(T x)
{
    uint64_t *s = slot[met[me]++ & 1], w = 0;
    memcpy(&w, &x, sizeof x);
    s[me] = w;
    if (_setjmp(at[me]) == 0) resume((me + 1) % N);
    return s;
}
template <typename T>
T as(uint64_t w)
{
    T x;
    memcpy(&x, &w, sizeof x);
    return x;
}
template <typename T>
T up(T x, int d)
{
    const uint64_t *s = exchange(x);
    return me >= d ? as<T>(s[me - d]) : x;
}
template <typename T>
T of_lane(T x, int lane)
{
    return as<T>(exchange(x)[lane]);
}
template <typename T>
T of_first(T x)
{
    const uint64_t *s = exchange(x);
    for (int i = 1; i < N; ++i) uneven += s[i] != s[0];     // (only what is the same in all lanes is asked for)
    return as<T>(s[0]);
}
static uint64_t ballot(bool x)
{
    const uint64_t *s = exchange((uint64_t)x);
    uint64_t m = 0;
    for (int i = 0; i < N; ++i) m |= s[i] << i;
    return m;
}
struct Thread { unsigned x; };
}  // namespace lanes
#define threadIdx (lanes::Thread{(unsigned)lanes::me})
#define __shfl_up lanes::up
#define __builtin_amdgcn_readlane lanes::of_lane
#define __builtin_amdgcn_readfirstlane lanes::of_first
#define __ballot lanes::ballot
#define __popcll __builtin_popcountll
static int min(int x, int y) { return x < y ? x : y; }
static int max(int x, int y) { return x > y ? x : y; }

#include "chunk_plan.h"

static ss::ChunkArgs args;
static int span_now;
static std::vector<int32_t> found;     // span, request, tile, from, to, place, pieces (0: not counted)

template <int ROWS, int KEYS, int OPEN>
static void walk()
{
    ss::ChunkWalk<ROWS, KEYS, OPEN> s;
    for (bool any = s.begin(args, span_now); any; any = s.next(args)) {
        const int count = s.part == 2 * span_now + 1 ? s.pieces() : 0;
        if (lanes::me == 0)
            for (int x : {span_now, s.b, s.t, s.s0, s.s1, s.part, count}) found.push_back(x);
    }
}
extern "C" const int32_t *plan(int f32, int batch, int max_blocks, int num_blocks, int total_rows, int hq, int hkv, int spans, const int32_t *kv_len, const int32_t *q_indptr,
                               int32_t *pieces)
{
    args = ss::ChunkArgs{};
    args.batch = batch;
    args.max_blocks = max_blocks;
    args.num_blocks = num_blocks;
    args.total_rows = total_rows;
    args.num_q_heads = hq;
    args.num_kv_heads = hkv;
    args.spans = spans;
    args.kv_len = kv_len;
    args.q_indptr = q_indptr;
    found.clear();
    lanes::uneven = 0;
    for (span_now = 0; span_now < spans; ++span_now)
        lanes::run(f32 ? walk<ss::kChunkRowsF32, ss::kChunkKeysF32, ss::kChunkOpenF32> : walk<ss::kChunkRows, ss::kChunkKeys, ss::kChunkOpen>);
    *pieces = lanes::uneven ? -1 : (int)found.size() / 7;
    return found.data();
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    d = tmp_path_factory.mktemp("chunk_plan")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-U_FORTIFY_SOURCE", "-D__HIP_PLATFORM_AMD__", "-shared", "-fPIC", "-isystem", os.path.join(ROCM, "include"),
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2604_09562_amd", "csrc"), str(d / "shim.cpp"), "-o", str(d / "shim.so")], check=True)
    lib = ctypes.CDLL(str(d / "shim.so"))
    lib.plan.restype = ctypes.POINTER(ctypes.c_int32)
    return lib


def walked(shim, f32, lengths, hq, hkv, spans, q_indptr=None, max_blocks=None, num_blocks=1 << 20, total_rows=None):
    """[(span, request, tile, from, to, place, pieces)]"""
    kv = np.array([n for _, n in lengths], np.int32)
    indptr = np.concatenate([[0], np.cumsum([q for q, _ in lengths])]).astype(np.int32) if q_indptr is None else np.array(q_indptr, np.int32)
    width = max([-(-int(n) // 16) for n in kv] + [1]) if max_blocks is None else max_blocks
    n, as_ints = ctypes.c_int32(), lambda a: a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))  # noqa: E731
    got = shim.plan(int(f32), len(lengths), width, num_blocks, int(indptr[-1]) if total_rows is None else total_rows, hq, hkv, spans, as_ints(kv), as_ints(indptr), ctypes.byref(n))
    assert n.value >= 0, "lanes that should agree do not"
    return [tuple(got[7 * i:7 * i + 7]) for i in range(n.value)]


def check(shim, f32, lengths, hq, hkv, spans):
    rows, keys, G = (64, 64, hq // hkv) if f32 else (256, 32, hq // hkv)
    label = (f32, lengths, hq, hkv, spans)
    tiles, places = {}, {}
    for span, b, t, s0, s1, place, count in walked(shim, f32, lengths, hq, hkv, spans):
        tiles.setdefault((b, t), []).append((span, s0, s1, place, count))
    for b, (q, n) in enumerate(lengths):
        for t in range(-(-q * G // rows)):
            last = min(((t + 1) * rows - 1) // G, q - 1)                  # the last of the tile's new tokens
            steps = max(0, -(-(n - q + last + 1) // keys))
            pieces = tiles.pop((b, t), None)
            assert pieces, (label, b, t, "no piece")
            assert [s0 for _, s0, _, _, _ in pieces] == [0] + [s1 for _, _, s1, _, _ in pieces[:-1]] and pieces[-1][2] == steps, (label, b, t, steps, pieces)
            first = pieces[0][0]
            if len(pieces) == 1:
                assert pieces[0][3] == -1, (label, b, t, pieces)
                continue
            assert pieces[0][4] == len(pieces), (label, b, t, f"{len(pieces)} pieces, counted as {pieces[0][4]}")
            assert [p[3] for p in pieces] == [2 * (first + i) + (i == 0) for i in range(len(pieces))], (label, b, t, pieces)
            for p in pieces:
                assert p[2] > p[1] and p[3] < 2 * spans and p[3] not in places, (label, b, t, pieces)
                places[p[3]] = (b, t)
    assert not tiles, (label, tiles)


@pytest.mark.parametrize("lengths,hq,hkv", [([(389, 489)], 32, 8), ([(385, 485)], 32, 8), ([(519, 519)], 8, 8), ([(521, 521)], 8, 8), ([(259, 259)], 16, 8), ([(1031, 1031)], 8, 8)])
def test_last_tiles_that_are_not_full(shim, lengths, hq, hkv):
    """The cost in front of a tile is interpolated between a request's first and last tile: a short last one leaves the others cheaper than they are."""
    check(shim, False, lengths, hq, hkv, 256 // hkv)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("G", [1, 2, 4, 5, 7, 8, 16])
def test_random_batches(shim, f32, G):
    rng = np.random.default_rng(100 * G + f32)
    for _ in range(60):
        hkv = int(rng.choice([1, 2, 4, 8]))
        batch = int(rng.choice([1, 1, 2, 3, 8, 70]))
        lengths = []
        for _ in range(batch):
            q = int(round(np.exp(rng.uniform(0, np.log(2000 if batch < 8 else 300)))))
            n = q + (int(np.exp(rng.uniform(0, np.log(20000)))) if rng.random() < 0.7 else 0)
            if rng.random() < 0.1:
                q, n = (0, n) if rng.random() < 0.5 else (q, int(rng.integers(0, q + 1)))   # no new tokens; a cache shorter than the rows
            lengths.append((q, n))
        spans = int(rng.choice([1, 2, 7, 256 // hkv, 256 // hkv, 512 // hkv]))
        check(shim, f32, lengths, hkv * G, hkv, spans)


@pytest.mark.parametrize("f32", [False, True])
def test_requests_whose_lengths_are_impossible_have_no_tiles(shim, f32):
    """Rows outside the call's or a cache longer than the table's row: no piece.  The others are cut as if those had no new tokens."""
    lengths = [(300, 700), (64, 64), (200, 900), (5, 90)]
    spans, big = 32, 2 ** 31 - 1
    for change in (lambda q, n: n.__setitem__(1, 16 * 57 + 1), lambda q, n: n.__setitem__(1, big), lambda q, n: q.__setitem__(slice(1, 3), [300, 299]),
                   lambda q, n: q.__setitem__(slice(1, 3), [-5, -2]), lambda q, n: q.__setitem__(slice(1, 3), [-big - 1, 5]),
                   lambda q, n: q.__setitem__(slice(1, 3), [5, -big]), lambda q, n: q.__setitem__(slice(2, 5), [570, 571, big])):
        indptr, kv = [0, 300, 364, 564, 569], [n for _, n in lengths]
        change(indptr, kv)
        got = walked(shim, f32, [(0, n) for n in kv], 8, 2, spans, q_indptr=indptr, max_blocks=57, total_rows=569)
        fits = [0 <= a <= b <= 569 and n <= 57 * 16 for a, b, n in zip(indptr, indptr[1:], kv)]
        assert not all(fits) and {b for _, b, *_ in got} <= {b for b in range(4) if fits[b] and indptr[b + 1] > indptr[b]}
        steps = {}
        for _, b, t, s0, s1, _, _ in got:
            steps[b, t] = steps.get((b, t), 0) + s1 - s0
        for (b, t), n in steps.items():
            rows, keys = (64, 64) if f32 else (256, 32)
            chunk = indptr[b + 1] - indptr[b]
            last = min(((t + 1) * rows - 1) // 4, chunk - 1)
            assert n == -(-(kv[b] - chunk + last + 1) // keys)
    assert walked(shim, f32, lengths, 8, 2, spans, num_blocks=0) == []           # no cache, no keys
    assert [p[3:6] for p in walked(shim, f32, [(3, -5), (2, -big - 1)], 8, 2, 1)] == [(0, 0, -1)] * 2   # (rows in front of the cache: nothing to see)
