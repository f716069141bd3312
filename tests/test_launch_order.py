"""CPU: what a kernel may read before its stream predecessor is over.

Kernels launched by locks_launch_pdl may start while the kernel before them still runs (several of them let their successor start at once),
and whatever that one writes is there only after pdl_wait().  The library's rotations and appends write the queries that attention and the
exact selector read, so no kernel reads device memory before its wait; and none reads it by the non-coherent path, which
is for what nobody writes while the kernel exists."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_24555_b200", "csrc")


def sources():
    return {os.path.basename(f): re.sub(r"//[^\n]*", "", open(f).read()) for f in sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh")))}


def body(text, at):
    """From the brace that opens at or after `at` to the one that closes it."""
    i = text.index("{", at)
    depth = 0
    for j in range(i, len(text)):
        depth += {"{": 1, "}": -1}.get(text[j], 0)
        if depth == 0:
            return text[i:j + 1]
    raise AssertionError("unbalanced braces")


def dependent_kernels():
    """(file, name, body) of every kernel that is launched so that it may start early."""
    text = sources()
    names = set()
    for t in text.values():
        for call in re.finditer(r"locks_launch_pdl(?:_cluster)?\(\s*([a-z_0-9]+)", t):
            names.add(call.group(1))
    names.discard("void")   # (the launchers' own declarations)
    found = []
    for f, t in text.items():
        for k in re.finditer(r"__global__\s+void\s+(?:__launch_bounds__\((?:[^()]|\([^()]*\))*\)\s*)?([a-z_0-9]+)\(", t):
            if k.group(1) in names:
                found.append((f, k.group(1), body(t, t.index(")", k.end()))))
    assert {n for _, n, _ in found} == names
    return found


def test_every_kernel_that_may_start_early_waits_before_it_reads():
    kernels = dependent_kernels()
    assert len(kernels) >= 14
    for f, name, b in kernels:
        assert "pdl_wait();" in b, (f, name)
        before = b[:b.index("pdl_wait();")]
        for reading in (r"__ldg\(", r"__ldcg\(", r"\bp\.\w+\s*\[", r"\w+r\[", r"\*\s*reinterpret_cast<const", r"cp_async", r"ld\.global"):
            got = re.search(reading, before)
            assert not got, (f, name, got.group(0))


def test_nothing_is_read_by_the_non_coherent_path():
    for f, t in sources().items():
        assert "__ldg(" not in t and "ld.global.nc" not in t, f


def test_tensor_memory_is_reached_by_whole_warps():
    """Tensor-memory loads and stores (and numbered barriers) are executed by all lanes of a warp together: wherever the chunk form
    branches by lane, the lanes come together before the next of them."""
    t = " ".join(sources()["kvq_chunk.cu"].split())
    for start in ("auto rescale = [&](float fix, int columns) {",                         # called where some row's maximum rose
                  "for (int c = 0; c < LOCKS_D; c += 32) { uint32_t s[32];",              # results: rows differ in what is not finite
                  "if (lane == 0) ms.red[8 * kv + warp - 8] = y; }"):
        at = t.index(start) + len(start)
        assert t[at:].lstrip().startswith("__syncwarp();"), start
    # where rows differ in what they see of a tile
    assert "decltype(masked_)::value; if (kMasked) __syncwarp();" in t and "if (kMasked) __syncwarp(); tmem_st<16>(w, " in t
    assert "if (part == 1 && i < 3) { if (kMasked) __syncwarp(); tmem_wait_ld();" in t
    assert re.search(r"if \(warp == 16\) \{ __syncwarp\(\); asm volatile\(\"tcgen05\.alloc", t)
    assert re.search(r"__syncwarp\(\); fence_after\(\); asm volatile\(\"tcgen05\.dealloc", t)
