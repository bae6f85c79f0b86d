"""How many merge blocks of the 4-bit attention share a multiprocessor: what the launch is made for has to fit its shared memory."""
import os
import re
import subprocess

from paper_2605_23258_b200 import build


def test_the_blocks_that_share_a_multiprocessor_fit(tmp_path):
    source = tmp_path / "blocks.cu"
    source.write_text("""#include "decode_q4.cuh"
using namespace vec::dq4;
template <typename T, int D, int THREADS> constexpr bool fits() {
    return merge_blocks<T, D, THREADS>() >= 1 && merge_blocks<T, D, THREADS>() * (MapTile<T, D>::BYTES + merge_shared<D>() + 1024) <= 228 * 1024 && merge_blocks<T, D, THREADS>() * THREADS <= 2048;
}
using B = __nv_bfloat16;
static_assert(fits<B, 64, MERGE_THREADS>() && fits<B, 128, MERGE_THREADS>() && fits<float, 64, MERGE_THREADS>() && fits<float, 128, MERGE_THREADS>());
static_assert(fits<B, 64, MERGE_MOST>() && fits<B, 128, MERGE_MOST>() && fits<float, 64, MERGE_MOST>() && fits<float, 128, MERGE_MOST>());
static_assert(merge_blocks<B, 128, MERGE_THREADS>() == 4 && merge_blocks<float, 64, MERGE_THREADS>() == 3 && merge_blocks<float, 128, MERGE_THREADS>() == 2);
template __global__ void vec::dq4::decode_q4_merge<float, 128, 4, MERGE_THREADS>(const unsigned char*, Cache, int, int, int, const float*, void*, int);
template __global__ void vec::dq4::decode_q4_merge<B, 64, 1, MERGE_MOST>(const unsigned char*, Cache, int, int, int, const B*, void*, int);
constexpr int shared[] = {merge_shared<128>(), merge_shared<64>()};
extern "C" const int* sizes() { return shared; }
""")
    done = subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-c", str(source), "-o", str(tmp_path / "blocks.o")], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert done.returncode == 0, done.stdout
    own = {int(d): int(n) for d, n in re.findall(r"Compiling entry function '\S*decode_q4_merge\S*Li(128|64)ELi\dE\S*'.*?(\d+) bytes smem", done.stdout, re.S)}
    count = lambda d: 2 * 8 * (d + 4) * 4 + 96 + 2 * 8 * 64 * 4 + 64 * 2 * 8 * 8  # noqa: E731
    assert {d: n <= count(d) for d, n in own.items()} == {128: True, 64: True}, own


def test_the_launch_goes_by_it():
    text = open(os.path.join(build.CSRC, "decode_q4.cu")).read()
    assert "merge_blocks<T, D, MERGE_THREADS>() * sm_count()" in text
