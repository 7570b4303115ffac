"""How many tiles of rows a workgroup of attention over the whole 8-bit cache takes, without a GPU: where one choice measured clearly
faster, it is the one that is made."""
import os
import subprocess

import pytest

import paper_2508_19740_amd as sp
from test_cache_host import CSRC, HEAD, ROOT

# batch, key-value heads, MB of codes, rows of a head, microseconds with one tile and with two (bfloat16 queries, E4M3, nothing in a cache)
MEASURED = [
    (8, 8, 4, 33, 8.9, 13.3), (8, 8, 4, 64, 9.0, 13.3), (1, 32, 4, 128, 10.2, 14.7), (1, 8, 4, 256, 16.6, 22.1), (1, 8, 4, 512, 17.2, 22.4),
    (1, 1, 1, 128, 19.5, 24.8), (1, 1, 4, 512, 48.1, 55.8), (8, 8, 8, 32, 11.0, 15.2), (8, 8, 8, 48, 10.8, 15.2), (1, 8, 8, 80, 19.4, 26.7),
    (8, 8, 16, 40, 14.3, 18.2), (1, 8, 16, 33, 18.0, 21.4), (1, 8, 16, 128, 23.8, 27.6), (1, 32, 32, 17, 18.4, 21.4), (1, 8, 64, 17, 25.4, 29.7),
    (1, 8, 64, 32, 26.4, 32.2), (16, 8, 32, 32, 18.7, 21.3), (1, 1, 128, 32, 40.8, 47.2), (1, 8, 128, 24, 38.1, 41.8), (8, 8, 192, 32, 47.2, 52.1),
    (8, 8, 384, 17, 85.0, 74.4), (8, 8, 512, 32, 112.2, 97.9), (1, 8, 512, 24, 110.0, 95.4), (8, 8, 128, 48, 51.0, 45.3), (8, 8, 256, 33, 92.0, 76.5),
    (1, 8, 512, 64, 172.5, 143.3), (1, 32, 64, 96, 47.7, 38.4), (1, 32, 96, 160, 94.5, 66.4), (1, 8, 64, 256, 79.1, 66.7), (8, 8, 32, 256, 47.5, 38.8),
    (1, 8, 128, 128, 84.5, 73.4), (1, 8, 16, 1024, 72.9, 60.5), (1, 1, 32, 512, 79.7, 65.8), (1, 1, 128, 2048, 2041.5, 836.6),
]

SOURCE = HEAD + r"""
#include <stdlib.h>
int main(int argc, char** argv)
{
    const int code = atoi(argv[1]);
    for (int i = 2; i + 3 < argc; i += 4) {
        const int B = atoi(argv[i]), H = atoi(argv[i + 1]), rows = atoi(argv[i + 3]);
        const long n = (static_cast<long>(atoi(argv[i + 2])) << 20) / (256L * B * H);
        const spotlight_config cfg = config(B, H, H, n > rows ? n : rows, 1);
        Plan p;
        cache::DensePlan d;
        if (make_plan(&cfg, &p) != SPOTLIGHT_OK || cache::plan_dense(p, 256, n, rows, nullptr, &d, code) != SPOTLIGHT_OK) return 2;
        printf("%d ", d.row_tiles);
        p.kv_dtype = SPOTLIGHT_F32;
        if (cache::plan_dense(p, 256, n, rows, nullptr, &d, code) != SPOTLIGHT_OK || d.row_tiles != 1) return 3;
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def chosen(tmp_path_factory):
    src = tmp_path_factory.mktemp("tiles") / "host.cpp"
    exe = str(src)[:-4]
    src.write_text(SOURCE)
    lib = sp.lib._name
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-w", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
                    "-I", CSRC, str(src), "-o", exe, lib, f"-Wl,-rpath,{os.path.dirname(lib)}", "-L/opt/rocm/lib",
                    "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"], check=True)

    def run(cells, code=sp.binding.E4M3):
        out = subprocess.run([exe, str(code), *(str(x) for c in cells for x in c)], capture_output=True, text=True)
        assert out.returncode == 0, out.returncode
        return [int(x) for x in out.stdout.split()]
    return run


def test_the_faster_kernel_is_chosen(chosen):
    got = chosen([c[:4] for c in MEASURED])
    slow = [(c, g) for c, g in zip(MEASURED, got) if (c[4] < c[5]) != (g == 1)]
    assert not slow, slow


def test_few_rows_and_borders(chosen):
    """16 rows never need a second tile; up to 32 rows the last-level cache's size decides (for integers, up to 24 rows, less), above
    that rows times bytes."""
    assert chosen([(1, 8, mb, 16) for mb in (1, 64, 512, 2048)]) == [1, 1, 1, 1]
    for rows in (17, 32):
        assert chosen([(1, 8, mb, rows) for mb in (16, 128, 129, 255, 256, 512)]) == [1, 1, 1, 1, 2, 2]
    for rows in (17, 24):
        assert chosen([(1, 8, mb, rows) for mb in (16, 64, 95, 96, 128, 129, 256, 512)], sp.binding.I8) == [1, 1, 1, 2, 2, 2, 2, 2]
    for rows in (25, 32):
        assert chosen([(1, 8, mb, rows) for mb in (16, 128, 129, 255, 256)], sp.binding.I8) == [1, 1, 1, 1, 2]
    assert chosen([(1, 8, 64, 47), (1, 8, 64, 48), (1, 8, 16, 191), (1, 8, 16, 192), (1, 8, 128, 33)]) == [1, 2, 1, 2, 2]
