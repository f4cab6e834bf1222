"""What no run shows: orders that a kernel's source has to ask the compiler for."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_18703_amd", "csrc")


def code(path):
    with open(path) as f:
        text = f.read()
    return re.sub(r"/\*.*?\*/|//[^\n]*", "", text, flags=re.S)


def test_barriers_order_memory():
    """The builtin of a barrier orders no memory for the compiler: LDS reads may be moved before it, where another wave's
    asynchronous loads have not arrived.  __syncthreads, or an asm statement that clobbers memory, does."""
    sources = glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h"))
    assert len(sources) > 15
    for path in sources:
        text = code(path)
        assert "__builtin_amdgcn_s_barrier" not in text, path
        for asm in re.findall(r"asm\b[^;]*s_barrier[^;]*;", text):
            assert '"memory"' in asm, (path, asm)


def test_lanes_of_a_wave_in_order():
    """A tile of a product leaves through LDS that its wave alone uses: what lanes write there others read, and write
    again.  Between each of these the source has to ask for the order."""
    text = code(os.path.join(CSRC, "k_project.hip"))
    text = text[text.index("void __launch_bounds__(kWavesN"):text.index("k_project_few")]
    at = 0
    for step in (r"scales\[i\] =", r"lanes_in_order\(\);", r"= \*\(const f32x4 \*\)\(scales", r"\*\(Vec4<T> \*\)\(room",
                 r"lanes_in_order\(\);", r"= \*\(const u32x4 \*\)\(room", r"= \*\(const T \*\)\(room", r"lanes_in_order\(\);\s*}\s*}"):
        found = re.search(step, text[at:])
        assert found, step
        at += found.end()
