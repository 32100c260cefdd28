"""The build refuses kernels that spill registers to scratch memory."""
import pytest

from paper_2608_14376_amd import build

KERNEL = """#include <hip/hip_runtime.h>
__global__ void k(float *p, int n)
{
    float a[ELEMS];
    for (int i = 0; i < ELEMS; ++i) a[i] = p[i * 64 + threadIdx.x];
    for (int i = 0; i < n; ++i) a[(i * 7) % ELEMS] += a[(i * 3) % ELEMS];
    for (int i = 0; i < ELEMS; ++i) p[i * 64 + threadIdx.x] = a[i];
}
"""


def test_remarks_name_the_kernels_with_scratch():
    remark = "x.hip:3:1: remark: %s [-Rpass-analysis=kernel-resource-usage]\n    3 | {\n      | ^\n"
    text = "".join(remark % ln for ln in (
        "Function Name: one", "    VGPRs: 20", "    ScratchSize [bytes/lane]: 0", "    VGPRs Spill: 0",
        "Function Name: two", "    VGPRs: 128", "    ScratchSize [bytes/lane]: 100", "    VGPRs Spill: 24"))
    assert build.scratch_of(text) == {"two": 100}
    assert build.scratch_of("") == {}


@pytest.mark.parametrize("elems,fine", [(1, True), (64, False)])
def test_a_kernel_with_scratch_does_not_build(tmp_path, elems, fine):
    src, obj = tmp_path / "k.hip", tmp_path / "k.o"
    src.write_text(KERNEL.replace("ELEMS", str(elems)))
    if fine:
        build.compile_object(str(src), str(obj))
        assert obj.exists()
    else:
        with pytest.raises(RuntimeError, match="scratch"):
            build.compile_object(str(src), str(obj))
