"""The launches of the block operators' calls, recorded on the CPU (see
block_recorder.c), with the library and with the one whose host code is built
with AddressSanitizer and UndefinedBehaviorSanitizer: batches, widths and
expert counts at the far end of what the calls accept, and the shapes that the
experts' layer takes."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = 0, 1


def _recorder(tmp_path_factory, lib, cc):
    libdir = os.path.dirname(lib)
    exe = str(tmp_path_factory.mktemp("rec") / "block_recorder")
    r = subprocess.run([*cc, "-std=gnu99", "-Wall", "-Werror", "-rdynamic", "-I", os.path.join(ROOT, "include"),
                        os.path.join(ROOT, "tests", "block_recorder.c"), "-o", exe, "-L", libdir,
                        "-l" + os.path.basename(lib)[3:-3], f"-Wl,-rpath,{libdir}",
                        "-Wl,--allow-shlib-undefined"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(lines):
        env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1")
        r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=120,
                           env=env)
        assert r.returncode == 0, r.stdout + r.stderr
        out = []
        for line in r.stdout.splitlines():
            st, *la = line.split()
            out.append((int(st), [tuple(int(v) for v in e.split(",")) for e in la]))
        assert len(out) == len(lines)
        return out
    return run


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not available")
    from paper_2603_04800_amd import _libpath
    return _recorder(tmp_path_factory, _libpath.LIB, [gcc])


MOST = 2 ** 31 - 1
FAR = [
    # (small GEMM tiles past 2^24 workgroups, the last rows of 32-bit counts)
    f"epilogue 67108860 16 16 0 1 {BF16} {BF16} 8 1", f"epilogue 33 16 1073741824 0 1 {BF16} {BF16} 8 0",
    f"epilogue 67108860 64 32 0 1 {BF16} {BF16} 4 17", f"epilogue 16 133136 4096 256 4 {F32} {F32} 8 18",
    f"epilogue 67000000 64 16 64 3 {BF16} {BF16} 8 2", "epilogue 1 64 1073741760 0 1 1 1 8 17",
    f"route {MOST} 512 1 {F32} 1", f"route {MOST // 16} 512 16 {BF16} 1", f"route {MOST // 8} 8 8 {BF16} 0",
    f"experts 67108860 67108860 1 16 16 0 1 {BF16} 8 1 0", f"experts 1 {MOST} 512 16 16 0 1 {F32} 8 0 1",
    f"experts 5 {MOST} 512 64 32 256 4 {BF16} 8 17 1", f"experts {MOST} {MOST} 2 64 16 64 2 {BF16} 4 0 0",
    f"experts 1 1 512 64 1073741824 16 2 {BF16} 8 0 1", f"experts 4096 500000000 1 64 512 16 2 {BF16} 8 17 1",
    f"combine {MOST} {MOST} 16 16 {BF16}", f"combine {2 ** 20} {MOST} 1073741824 1 {F32}",
]


@pytest.mark.parametrize("call", FAR)
def test_launches_stay_within_the_thread_limit(record, call):
    status, launches = record([call])[0]
    assert status == 0 and launches, (call, status, launches)


@pytest.mark.parametrize("call,launches", [
    # fp32 factors and ranks past 64: one launch before the product, also where
    # both of its roles together pass one launch dimension
    (f"epilogue 67000000 64 16 256 2 {F32} {F32} 8 0", 2), (f"epilogue 67108860 16 16 64 4 {BF16} {F32} 8 0", 2),
    (f"epilogue 67108860 64 32 128 2 {BF16} {BF16} 4 17", 2), (f"epilogue 333 1040 2000 16 2 {F32} {F32} 8 2", 2),
    # a split K and a long walk: the layer's own quantisation and down-projection
    (f"epilogue 20 18944 1024 64 2 {F32} {F32} 8 0", 3),
])
def test_first_stage_of_fp32_factors_and_high_ranks(record, call, launches):
    status, la = record([call])[0]
    assert status == 0 and len(la) == launches, (call, status, la)
    for x, y, z, threads in la:
        assert x * threads < 2 ** 32 and y * z < 2 ** 16 and x * y * z > 0


def test_host_code_under_sanitizers(tmp_path_factory):
    clang = "/opt/rocm/llvm/bin/clang"
    if not os.path.exists(clang):
        pytest.skip("ROCm clang not available")
    from paper_2603_04800_amd import build
    run = _recorder(tmp_path_factory, build.build_sanitized(),
                    [clang, "-fsanitize=address,undefined", "-fno-sanitize-recover=all"])
    bad = ["epilogue 4 64 48 0 1 1 1 8 17", "epilogue 4 64 64 0 1 1 1 8 -5", "epilogue -1 64 64 0 1 1 1 8 0",
           "epilogue 4 64 64 0 1 1 1 2147483647 0", "route -1 8 2 1 0", "route 4 8 9 1 0", f"route {MOST} 512 2 1 0",
           "experts 4 -8 4 64 64 0 1 1 8 0 1", "experts 4 8 0 64 64 0 1 1 8 0 1", f"experts 4 {MOST} 8 64 1073741824 0 1 1 8 0 1",
           "experts 4 8 4 64 64 0 1 1 8 0 0", "combine 4 8 24 2 1", "combine 4 -8 64 2 1"]
    good = FAR + ["epilogue 0 64 64 16 2 1 1 8 0", "route 0 8 2 1 1", "experts 0 0 4 64 64 0 1 1 8 0 1",
                  "combine 0 8 64 2 1"]
    out = run(bad + good)
    assert all(st > 0 and not la for st, la in out[:len(bad)]), out[:len(bad)]
    assert all(st == 0 for st, _ in out[len(bad):]), out[len(bad):]


def test_launches_of_a_call(record):
    """Few launches: one of routing up to 64 tokens, two up to 8192, three past
    them; two of the experts' layer, with and without a compensation."""
    one, two, three = record(["route 64 128 8 1 1", "route 8192 128 8 1 1", "route 8193 128 8 1 1"])
    assert (len(one[1]), len(two[1]), len(three[1])) == (1, 2, 3)
    for st, la in record(["experts 9 72 64 2048 2048 32 2 1 8 17 1", "experts 9 72 64 2048 2048 0 1 1 4 17 1",
                          "experts 4096 32768 64 2048 2816 32 2 1 8 17 1"]):
        assert st == 0 and len(la) == 2
    assert record(["combine 16 128 2048 8 1"])[0] == (0, [(16, 1, 1, 256)])


@pytest.mark.parametrize("n,E,K,N,bits,threads", [
    # few rows an expert: 32 x 64 tiles, two waves a block; more with packed weights
    (512, 64, 2048, 2048, 8, 256), (2048, 64, 2048, 2048, 4, 256),
    # 64 x 64 and 128 x 128 tiles have 256 threads as well, 256 x 256 have 512
    (4096, 64, 2048, 2048, 8, 256), (8192, 64, 2048, 2048, 8, 256),
    (32768, 64, 2048, 2816, 8, 512), (32768, 64, 2032, 2816, 8, 256), (2000, 2, 2048, 512, 8, 256),
])
def test_tile_shapes_of_the_experts(record, n, E, K, N, bits, threads):
    (st, launches), = record([f"experts 4096 {n} {E} {K} {N} 32 2 {BF16} {bits} 0 1"])
    assert st == 0 and launches[-1][3] == threads, launches
