"""Which kernel takes a call of wide trees' attention: the rule, compiled for the host."""
import ctypes
import subprocess

import pytest

from .helpers import CSRC


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule")
    (d / "r.cpp").write_text('#include "tree_rule.h"\n'
                             'extern "C" void rule(int b, int h, long long rows, long long keys, int dim, int kv8, int cus, int *o)\n'
                             '{\n    const ss::TreeUnitChoice c = ss::tree_unit_rule(b, h, rows, keys, dim, kv8 != 0, cus);\n    o[0] = c.tiles;\n    o[1] = c.splits;\n}\n'
                             'extern "C" int rule_f32(int b, int h, long long rows, long long keys, int dim, int cus) { return ss::tree_unit_f32_rule(b, h, rows, keys, dim, cus); }\n')
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    fn = ctypes.CDLL(str(d / "r.so")).rule
    fn.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_longlong, ctypes.c_longlong] + [ctypes.c_int] * 3 + [ctypes.c_void_p]

    def call(batch, heads, rows, keys, dim=128, kv8=False, cus=256):
        o = (ctypes.c_int * 2)()
        fn(batch, heads, rows, keys, dim, int(kv8), cus, o)
        return o[0], o[1]
    call.f32 = lambda batch, heads, rows, keys, dim=128, cus=256: ctypes.CDLL(str(d / "r.so")).rule_f32(
        batch, heads, ctypes.c_longlong(rows), ctypes.c_longlong(keys), dim, cus)
    return call


def test_short_calls_have_a_kernel_of_their_own(rule):
    assert rule(1, 8, 100, 336) == (4, 1)
    assert rule(1, 8, 100, 10000)[1] > 1 and rule(4, 2, 40, 64, 64) == (2, 1)
    assert rule(16, 8, 256, 8192)[0] == 0 and rule(8, 8, 480, 16384, kv8=True)[0] == 0 and rule(64, 8, 256, 1024)[0] == 0


@pytest.mark.parametrize("dim,kv8", [(128, False), (128, True), (64, False), (64, True)])
def test_cuts_of_any_call(rule, dim, kv8):
    """Tiles cover the widest tree, splits are at least eight steps, and a grid stays small, whatever the sizes."""
    for batch in (0, 1, 3, 64, 5000, 2 ** 31 - 1):
        for heads in (1, 2, 8, 128):
            for rows in (0, 1, 31, 32, 33, 100, 4096, 2 ** 31 - 1):
                for keys in (0, 16, 500, 70000, 2 ** 31 - 16):
                    if batch * heads > 2 ** 31:
                        continue
                    tiles, splits = rule(batch, heads, rows, keys, dim, kv8)
                    if tiles == 0:
                        continue
                    assert rows > 0 and tiles == -(-rows // 32) and splits in (1, 2, 4, 8, 16)
                    assert splits == 1 or -(-keys // 32) >= 8 * splits
                    assert tiles * batch * heads <= 65536
    assert rule(1, 8, 0, 100, dim, kv8) == (0, 1)


def test_short_calls_in_fp32(rule):
    assert rule.f32(4, 2, 160, 560, 64) == 10 and rule.f32(1, 8, 100, 336) == 7 and rule.f32(2, 8, 24, 300) == 2
    assert rule.f32(2, 2, 100, 10000, 64) == 0 and rule.f32(16, 8, 256, 364) == 0 and rule.f32(64, 8, 600, 450) == 0


@pytest.mark.parametrize("dim", [64, 128])
def test_cuts_of_any_call_in_fp32(rule, dim):
    for batch in (0, 1, 3, 64, 5000, 2 ** 31 - 1):
        for heads in (1, 2, 8, 128):
            for rows in (0, 1, 15, 16, 17, 100, 4096, 2 ** 31 - 1):
                for keys in (0, 16, 500, 70000, 2 ** 31 - 16):
                    if batch * heads > 2 ** 31:
                        continue
                    tiles = rule.f32(batch, heads, rows, keys, dim)
                    assert tiles == 0 or (rows > 0 and tiles == -(-rows // 16) and tiles * batch * heads <= 65536)
