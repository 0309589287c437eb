"""What the kernels of attention among a history's items ask for, from the metadata of the built library's code objects."""
from test_kernel_resources_cpu import scratch   # noqa: F401 (a fixture)

# bytes of scratch a lane, known and measured beside their dispatch: dk and dv of width 128 where the waves of a workgroup share its items
KNOWN = {"history_dkv_f32_kernelILi128ELb1E": 296, "history_dkv_kernelILi128ELi2ELi4E": 24}


def test_which_kernels_use_scratch(scratch):
    kernels = {k: n for k, n in scratch.items() if "5laser" in k and any(name in k for name in ("history_", "cache_"))}
    assert len(kernels) > 40
    spills = {k: n for k, n in kernels.items() if n}
    print(spills)
    assert len(spills) <= len(KNOWN)
    for k, n in spills.items():
        assert any(name in k and n <= most for name, most in KNOWN.items()), (k, n)
