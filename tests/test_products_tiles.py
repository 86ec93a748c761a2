"""Which shape of tile a product takes, without a device: a library in front of the runtime's looks at which kernel is launched."""
import products_tiles
import test_host_launches as host

NAMES = r"""
struct { const void *f; const char *name; } kernels[4096];
int n_kernels;
const char *launched = "";
void __hipRegisterFunction(void **modules, const void *f, char *stub, const char *name, unsigned limit, void *tid, void *bid, void *block, void *grid, int *size)
{
    if (strstr(name, "ecfm_") && n_kernels < 4096) kernels[n_kernels].f = f, kernels[n_kernels++].name = name;
}
static void note(const void *f)
{
    for (int i = 0; i < n_kernels; i++) if (kernels[i].f == f) launched = kernels[i].name;
}
"""

CODE = r"""
import re
sys.path.insert(0, "tests")
import products_tiles as sizes
from paper_2510_02676_amd import ecfa, ecfm
at, lib = 1 << 20, ecfm._lib                                            # an address that nothing looks at
def shape(rc):
    kind, args = re.search(r"ecfm_(few|many)_kernelI((?:L[ij]\d+E)+)", ctypes.c_char_p.in_dll(shim, "launched").value.decode()).groups()
    v = [int(x) for x in re.findall(r"L[ij](\d+)E", args)]
    assert rc == 0
    return (16 * v[1], 16 * v[0]) if kind == "few" else (v[0], v[1])
def operands(m, n, k, experts):
    return ecfm._Weights(at, at, k, n * k, n, k, experts, 0), ecfm._X(at, at, k, m, 1), ecfm._Y(at, n, m, ecfa.BF16)
for want, m, n, k in sizes.DENSE:
    w, x, y = operands(m, n, k, 1)
    assert shape(lib.ecfm_gemm(w, x, y, None)) == want, (want, m, n, k)
    assert m <= 16 or sizes.tiles(want, [m], n) > 256, (want, m, n, k)
def of_experts(m, n, k, experts):
    w, x, y = operands(m, n, k, experts)
    return shape(lib.ecfm_gemm_experts(w, at, x, at, y, None))
for want, counts, n, k in sizes.FEW:
    assert of_experts(sum(counts), n, k, len(counts)) == want, (want, counts, n, k)
for want, m, experts, unlike, n, k in sizes.MANY:
    assert of_experts(m, n, k, experts) == want and sizes.tiles(want, sizes.counts_of(m, experts, unlike), n) > 256, (want, m, experts, n, k)
"""


def test_shapes(tmp_path, monkeypatch):
    shim = host.SHIM.replace("hipError_t hipLaunchKernel(", NAMES + "hipError_t hipLaunchKernel(").replace("    return launches++", "    note(f);\n    return launches++")
    assert shim.count("note(f)") == 1
    monkeypatch.setattr(host, "SHIM", shim)
    host.run_on_shim(tmp_path, CODE)


def test_what_the_sizes_reach():
    """The shapes that take many tiles a workgroup have K of as few blocks as they take many tiles at, of one and two rounds of scales, and more."""
    blocks = {shape: sorted(-(-k // 128) for s, *_, k in products_tiles.MANY if s == shape) for shape in ((64, 128), (128, 128))}
    assert blocks[64, 128][0] == 10 and blocks[128, 128][0] == 3 and all(b[-1] > 16 for b in blocks.values())
