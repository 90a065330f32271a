"""Which kernels the linear layers' forward pass launches (host code, compiled here without a GPU): a product whose K is cut into
pieces goes by the kernel that knows pieces, one workgroup each at least, and is joined; no other is."""
import os
import random
import re
import subprocess

import pytest

from paper_1702_02181_amd import build_lib as B

# linear.hip with its launches written down instead of made
MAIN = r'''
#include <hip/hip_runtime.h>
#include <cstdio>
#include <string>
static std::string g_log;
static void note(const char* kernel, dim3 grid) { g_log += " " + std::string(kernel).substr(0, 17) + ":" + std::to_string(grid.x); }
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, ...) note(#kernel, grid)
#include "linear.hip"
fold::ProfScope::ProfScope(const char*, hipStream_t) {}
fold::ProfScope::~ProfScope() {}
int main() {
  int dtype, K, N;
  long long M;
  char* p = reinterpret_cast<char*>(4096);
  while (std::scanf("%d %lld %d %d", &dtype, &M, &K, &N) == 4) {
    g_log.clear();
    fold::launch_linear(dtype, M, K, N, p, p, nullptr, FOLD_ACT_GELU, nullptr, p, nullptr, p, nullptr);
    const fold::Shape s = fold::forward_shape(M, K, N, dtype == FOLD_BF16 ? 2 : 4);
    std::printf("%d %d %lld%s\n", s.wm, s.split, (long long)(s.mt * s.nt), g_log.c_str());
  }
}
'''


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    d = tmp_path_factory.mktemp("linear")
    (d / "main.hip").write_text(MAIN)
    r = subprocess.run([B.HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-I" + B.CSRC,
                        "-I" + os.path.join(B.ROOT, "include"), str(d / "main.hip"), "-Wl,--unresolved-symbols=ignore-all",
                        "-o", str(d / "launches")], capture_output=True, text=True)  # (the device code is left out)
    assert r.returncode == 0, r.stderr[-3000:]

    def run(sizes):
        text = "\n".join(" ".join(map(str, x)) for x in sizes)
        out = subprocess.run([str(d / "launches")], input=text, capture_output=True, text=True, check=True).stdout
        lines = out.splitlines()
        assert len(lines) == len(sizes)
        for line in lines:
            head = re.match(r"(\d+) (\d+) (\d+)", line)
            yield tuple(map(int, head.groups())), re.findall(r"(\w+)[^:]*:(\d+)", line[head.end():])
    return run


# layers whose 256 x 256 tiles are more than the compute units and whose K is long
LONG = [(1, m, k, n) for k, n, rows in
        ((16384, 4096, (4097, 5000, 5109, 5121, 6144, 8193, 10240, 12289, 14336, 16385, 17438)),
         (10240, 2560, (8193, 9728, 14721, 16384)), (8192, 2048, (10241, 10300, 10511)), (16000, 4099, (4200,)),
         (15012, 674, (43853,))) for m in rows]


def test_cut_products_go_by_the_kernel_that_knows_pieces(launches):
    rng = random.Random(1)
    drawn = [(rng.randrange(2), int(2 ** rng.uniform(6, 17)), int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 14)))
             for _ in range(20000)]
    cut = chains = 0
    for size, ((wm, split, tiles), made) in zip(LONG + drawn, launches(LONG + drawn)):
        if [k for k, _ in made] == ["kernel"]:  # few rows
            assert size[1] <= 64
            continue
        names = [k for k, _ in made]
        assert names[0] in ("k_product", "k_product_chain") and names[1:] == (["k_linear_join"] if split > 1 else []), (size, made)
        if names[0] == "k_product_chain":
            assert wm == 4 and split == 1 and tiles > 256, size
        else:
            assert int(made[0][1]) >= tiles * split, size
        cut, chains = cut + (split > 1), chains + (names[0] == "k_product_chain")
    assert cut > 500 and chains > 500  # both are drawn


def test_gradient_before_the_activation_alone_is_checked():
    """Asked for by itself it is an output like the others."""
    from paper_1702_02181_amd import fold as F
    from tests.test_oracle_vocab import NULL_STREAM, _Buf
    x, W, z, d, ws = (_Buf(1 << (20 + k)) for k in range(5))
    for kw in (dict(dpre=x), dict(dpre=_Buf(z.at + 16)), dict(dout=None), dict(pre=None)):
        a = dict(pre=z, dout=d, dpre=z)
        a.update(kw)
        with pytest.raises(F.FoldError) as e:
            F.fold_linear_backward(0, 4, 100, 70, x, W, F.FOLD_ACT_TANH, a["pre"], a["dout"], a["dpre"], 0, None, 0, None, None, 0,
                                   ws, 1 << 20, NULL_STREAM)
        assert e.value.code == F.FOLD_E_INVALID
