"""What the launches of the 4-bit layers ask of the runtime is shared by all host threads, and what a failed call leaves behind is seen by
the same thread's next one: looked at in the source (the threads themselves: test_gpu_group_threads.py)."""
import os
import re

GROUP = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2311_15806_b200", "csrc", "group")


def _sources():
    for name in sorted(os.listdir(GROUP)):
        if name.endswith((".cu", ".cuh")):
            yield name, re.sub(r"//[^\n]*", "", open(os.path.join(GROUP, name)).read())


def test_a_limit_of_a_kernel_is_set_once_to_its_most():
    calls = [(name, m) for name, text in _sources() for m in re.findall(r"cudaFuncSetAttribute\([^;]*;", text)]
    assert len(calls) == 1 and calls[0][0] == "group_entry.cu" and "MaxDynamicSharedMemorySize, most)" in calls[0][1]
    asked = [m for name, text in _sources() for m in re.findall(r"allow_dynamic_smem\(reinterpret_cast<const void\*>\(\w+\), ([^)]*)\)", text)]
    assert sorted(asked) == ["32 * PIPE_MAX_EXPERTS * 4", "kTMaxSmem"]   # (constants: no call's own size)


def test_a_failed_call_leaves_no_error_to_the_next_one():
    found = 0
    for name, text in _sources():
        for m in re.finditer(r"return PIPE_ERR_CUDA;", text):
            found += 1
            assert text[:m.start()].rstrip().endswith("cudaGetLastError();"), name
    assert found == 1
