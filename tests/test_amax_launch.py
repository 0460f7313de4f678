"""How a kernel behind an amax is launched, with the runtime's calls replaced at link time: needs no GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include "elementwise.cuh"

struct P { unsigned int *amax; };
template <int N> __global__ void kernel(const P p, int n) {}

namespace fp8dpa {
void set_error(const char *fmt, ...) { va_list ap; va_start(ap, fmt); vprintf(fmt, ap); va_end(ap); printf("; "); }
}
static unsigned largest;             // the largest cluster that the device can hold
extern "C" {
cudaError_t __wrap_cudaGetDevice(int *d) { *d = 0; return cudaSuccess; }
cudaError_t __wrap_cudaGetLastError(void) { return cudaSuccess; }
cudaError_t __wrap_cudaFuncSetAttribute(const void *, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t __wrap_cudaMemsetAsync(void *, int, size_t, cudaStream_t) { printf("memset "); return cudaSuccess; }
cudaError_t __wrap_cudaOccupancyMaxActiveClusters(int *n, const void *, const cudaLaunchConfig_t *c)
{
    const unsigned size = c->attrs[0].val.clusterDim.x;
    printf("ask(%u,%u,%zu) ", size, c->blockDim.x, c->dynamicSmemBytes);
    *n = size <= largest ? 1 : 0;
    return cudaSuccess;
}
cudaError_t __wrap_cudaLaunchKernel(const void *, dim3 g, dim3, void **, size_t, cudaStream_t) { printf("plain(%u) ", g.x); return cudaSuccess; }
cudaError_t __wrap_cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *, void **)
{
    const bool cluster = c->attrs[0].id == cudaLaunchAttributeClusterDimension;
    printf(cluster ? "cluster(%u) " : "early(%u) ", c->gridDim.x);
    return cluster && c->attrs[0].val.clusterDim.x > largest ? cudaErrorInvalidClusterSize : cudaSuccess;
}
}

int main(int argc, char **argv)
{
    static unsigned int amax;
    largest = atoi(argv[1]);
    const P p = {&amax};
    for (int i = 2; i + 1 < argc; i += 2) {
        const unsigned grid = atoi(argv[i]), threads = atoi(argv[i + 1]);
        printf("%d\n", fp8dpa::launch_behind_amax<kernel<0>>(1000, p.amax, grid, threads, 1024, 0, p, 1));
    }
    return 0;
}
"""
WRAPPED = ["cudaGetDevice", "cudaGetLastError", "cudaFuncSetAttribute", "cudaMemsetAsync", "cudaOccupancyMaxActiveClusters",
           "cudaLaunchKernel", "cudaLaunchKernelExC"]


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    d = tmp_path_factory.mktemp("launch")
    src, exe = d / "launch.cu", d / "launch"
    src.write_text(PROGRAM)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-cudart", "static", "-I",
                    os.path.join(ROOT, "paper_2505_20524_b200", "csrc"), str(src), "-o", str(exe)]
                   + [a for w in WRAPPED for a in ("-Xlinker", f"--wrap={w}")], check=True)

    def run(largest, *calls):
        out = subprocess.run([str(exe), str(largest)] + [str(v) for c in calls for v in c], check=True, capture_output=True, text=True)
        return out.stdout.strip().split("\n")

    return run


def test_small_grids_are_one_cluster(launches):
    got = launches(16, (2, 256), (8, 512), (9, 256), (16, 128), (16, 256))
    assert [g.split()[-2:] for g in got] == [["cluster(2)", "0"], ["cluster(8)", "0"], ["cluster(9)", "0"], ["cluster(16)", "0"], ["cluster(16)", "0"]]
    assert not any("memset" in g or "plain" in g for g in got)


def test_other_grids_stand_behind_a_memset(launches):
    assert launches(16, (17, 256), (9, 512), (1, 256)) == ["memset plain(17) 0", "memset plain(9) 0", "plain(1) 0"]


@pytest.mark.parametrize("largest", [8, 12, 15])
def test_a_device_without_clusters_of_16_gets_the_memset_form(launches, largest):
    """Where no cluster of 16 fits, a grid of 9 to 16 CTAs goes the way of one of 17; the runtime is asked once."""
    got = launches(largest, (9, 256), (16, 256), (13, 128), (8, 256))
    assert [g.split()[-1] for g in got] == ["0"] * 4
    assert [g.split()[-3:-1] for g in got[:3]] == [["memset", "plain(9)"], ["memset", "plain(16)"], ["memset", "plain(13)"]]
    assert got[3] == "cluster(8) 0" and "ask" not in "".join(got[1:])
