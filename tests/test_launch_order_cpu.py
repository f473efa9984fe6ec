"""Dependent launches: a kernel that takes tensor memory lets the next one begin only when it has it.  A block of the next
kernel on the same SM takes its own before it waits for the first kernel's end, and an allocation waits without a limit."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_27258_gb300", "csrc")


def kernels():
    """(file, name, body) of each kernel."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"__global__", text):
            at = text.index(") {", m.start()) + 2
            depth, end = 0, at
            while True:
                depth += {"{": 1, "}": -1}.get(text[end], 0)
                end += 1
                if depth == 0:
                    break
            head = re.sub(r"__launch_bounds__\((?:[^()]|\([^()]*\))*\)", "", text[m.start():at])
            yield os.path.basename(path), re.search(r"(\w+)\s*\(", head).group(1), text[at:end]


def test_tensor_memory_before_the_next_kernel():
    seen = []
    for path, name, body in kernels():
        took, let = [body.find(s) for s in ("tmem_alloc(", "tcgen05.alloc")], body.find("let_next_begin(")
        took = max(took)
        if took < 0 or let < 0:
            continue
        # behind the barrier that the allocating warp arrives at
        assert body.find("__syncthreads()", took) < let, (path, name)
        assert took < let, (path, name)
        seen.append(name)
    assert sorted(seen) == ["ffn_few_kernel", "ffn_tile_kernel", "ssm_state_kernel", "ssm_tc_kernel"]


def test_every_kernel_is_seen():
    names = [name for _, name, _ in kernels()]
    count = sum(open(p).read().count("__global__") for p in glob.glob(os.path.join(CSRC, "*.cu")))
    assert len(names) == count > 40 and {"bwd_tc_kernel", "hla2_fused_kernel", "glr_step_kernel"} <= set(names), names
