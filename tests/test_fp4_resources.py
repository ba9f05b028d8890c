"""The built library's 4-bit kernels and page bookkeeping, read on the CPU (nothing is launched): LDS against what a gfx950
CU holds, where matrix products leave their results, and what the other caches' kernels do not carry."""
import os
import re
import subprocess

import pytest

from paper_2504_15930_amd import build, sl
from test_kernel_resources import LDS_PER_CU, _code_objects, sizes, static_lds   # noqa: F401 (fixtures)
from test_matrix_waits import early_reads


def _lds(static_lds, name, count):
    hits = {k: v for k, v in static_lds.items() if name in k}
    assert len(hits) == count, (name, sorted(static_lds))
    return max(hits.values())


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    """The disassembly of every kernel, by mangled name."""
    objdump = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
    if not os.path.exists(objdump):
        pytest.skip("no llvm-objdump under ROCm here")
    if not os.path.exists(sl.LIBRARY):
        build.build()
    d, out = tmp_path_factory.mktemp("elf"), {}
    for i, elf in enumerate(_code_objects(open(sl.LIBRARY, "rb").read())):
        path = d / f"{i}.elf"
        path.write_bytes(elf)
        text = subprocess.run([objdump, "-d", str(path)], capture_output=True, text=True, check=True).stdout
        out.update(re.findall(r"^[0-9a-f]+ <(\S+)>:\n(.*?)(?=^[0-9a-f]+ <|\Z)", text, re.S | re.M))
    return out


# (two of head_dim 64 and two of 128: up to eight query heads per KV head, and more)
def test_split_kernels_fit_the_largest_batch(static_lds, sizes):
    assert _lds(static_lds, "split_fp4_kernel", 4) + sizes.split_bytes(sizes.max_batch(0)) <= LDS_PER_CU


def test_prefix_kernels_fit_every_accepted_size(static_lds, sizes):
    """Up to 4096 sequences in up to 4096 groups, 1 to 16 heads per KV head."""
    static, B = _lds(static_lds, "prefix_fp4_kernel", 4), sizes.max_batch(1)
    worst = max(sizes.prefix_bytes(B, ng, g) for ng in range(B + 1) for g in (1, 4, 5, 16))
    assert static + worst <= LDS_PER_CU, (static, worst)


@pytest.mark.parametrize("batch,groups,group", [(1536, 768, 7), (3000, 2, 7), (2700, 1, 16), (1000, 1000, 1)])
def test_two_prefix_workgroups_per_cu(static_lds, sizes, batch, groups, group):
    """The shared pages stream beside the own ones."""
    assert 2 * (_lds(static_lds, "prefix_fp4_kernel", 4) + sizes.prefix_bytes(batch, groups, group)) <= LDS_PER_CU


def test_two_split_workgroups_per_cu(static_lds, sizes):
    """The default with head_dim 64 and more than 128 sequences x KV heads."""
    hits = {k: v for k, v in static_lds.items() if "split_fp4_kernelILi64E" in k}
    assert len(hits) == 2 and all(2 * (v + sizes.split_bytes(1024)) <= LDS_PER_CU for v in hits.values())


def test_page_kernels_fit_the_largest_batch(static_lds, sizes):
    """Three numbers per request, and two more (extend_pages_kernel; the others hold fewer)."""
    B = sizes.max_batch(0)
    for name, count in (("extend_pages_kernel", 2), ("release_pages_kernel", 2), ("fill_slots_kernel", 1)):
        assert _lds(static_lds, name, count) + 4 * (3 * B + 2) <= LDS_PER_CU


@pytest.mark.parametrize("D", [64, 128])
def test_the_other_caches_merge_does_not_count_4_bit_workers(listings, D):
    """The prefix merge of a 4-bit cache looks up its shared-page workers; the bf16 and E4M3 caches' has no code for it."""
    size = {fp4: len([k for n, b in listings.items() if f"merge_prefix_kernelILi{D}ELb{fp4}E" in n for k in b.splitlines()])
            for fp4 in (0, 1)}
    assert 0 < size[0] < size[1]


def test_products_leave_their_results_in_ordinary_registers(listings):
    """The check of the wait states after matrix products (test_matrix_waits.py) follows v registers: no result may be in
    an accumulation register, whose readers it would not see. (The compiler may move other values there and back.)"""
    seen = 0
    for name, body in listings.items():
        for operands in re.findall(r"^\s+v_s?mfma\S* (.*?)\s*//", body, re.M):
            seen += 1
            assert re.fullmatch(r"v\[\d+:\d+\]", operands.split(", ")[0]), (name, operands)
    assert seen > 100


def test_products_of_every_kernel_are_read_after_their_wait(listings):
    """The other caches' kernels too."""
    kernels = {name: body for name, body in listings.items() if "v_mfma" in body}
    assert {k for k in ("split_kv_kernel", "prefix_split_kernel", "split_fp4_kernel", "prefix_fp4_kernel", "unit_fp4_kernel")
            if any(k in name for name in kernels)} == {"split_kv_kernel", "prefix_split_kernel", "split_fp4_kernel",
                                                       "prefix_fp4_kernel", "unit_fp4_kernel"}
    for name, body in kernels.items():
        assert not early_reads(body), name
