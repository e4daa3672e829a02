"""Every kernel instantiation compiled into libsparrow_paged.so and the GPU test that runs it against the formulas: the keys must be exactly the
`__global__` instantiations the library holds, and every test named must exist.  That each runs in the paged GPU tests was observed with a
kernel trace (profiles/paged_gpu_test_kernel_coverage.txt)."""
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2602_15318_amd", "libsparrow_paged.so")

PG, RP, CA = "test_gpu_paged_pages.py", "test_gpu_paged_rope.py", "test_gpu_chunk_attn.py"
COVERAGE = {
    "page_update_kernel<true>": (PG, "test_grow_and_roll_back"),
    "page_update_kernel<false>": (PG, "test_long_prompts"),
    "page_rows_kernel": (PG, "test_long_prompts"),
    **{f"mrope_table_kernel<{d}>": (RP, "test_table") for d in (64, 128)},
    **{f"mrope_append_kernel<{t}, {d}>": (RP, "test_append") for t in ("float", "unsigned short") for d in (64, 128)},
    # bf16, more than 64 rows (new token, query head of the group) per KV head
    **{f"chunk_many_kernel<{d}>": (CA, "test_chunks") for d in (64, 128)},
    # <head_dim, 32-row tiles>: 17 to 32 and 33 to 64 rows
    **{f"chunk_few32_kernel<{d}, {rt}>": (CA, "test_few_tokens_each") for d in (64, 128) for rt in (1, 2)},
    # <storage type, head_dim, 16-row tiles, wavefronts>
    **{f"chunk_few16_kernel<float, {d}, {rt}, 4>": (CA, "test_few_tokens_each") for d in (64, 128) for rt in (1, 2)},
    **{f"chunk_few16_kernel<unsigned short, {d}, 1, {w}>": (CA, "test_pieces_put_together") for d in (64, 128) for w in (2, 4, 8)},
    # fp32, more than 32 rows
    **{f"chunk_f32_kernel<{d}>": (CA, "test_chunks") for d in (64, 128)},
    # <storage type, head_dim, wavefronts that share a row's pieces>
    **{f"chunk_combine_kernel<{t}, {d}, {n}>": (CA, "test_pieces_put_together") for t in ("float", "unsigned short") for d in (64, 128)
       for n in (1, 2, 8)},
}


def test_every_compiled_kernel_instantiation_has_a_test():
    if not os.path.exists(LIB):
        from paper_2602_15318_amd import build
        build.build()
    out = subprocess.run(["nm", "-C", LIB], capture_output=True, text=True, check=True).stdout
    compiled = set(re.findall(r"__device_stub__(.*?)\(", out))
    assert compiled == set(COVERAGE), (sorted(compiled - set(COVERAGE)), sorted(set(COVERAGE) - compiled))


def test_the_named_tests_exist_and_the_trace_has_them():
    trace = open(os.path.join(ROOT, "profiles", "paged_gpu_test_kernel_coverage.txt")).read()
    for kernel, (fname, test) in COVERAGE.items():
        src = open(os.path.join(ROOT, "tests", fname)).read()
        assert re.search(rf"^def {test}\(", src, flags=re.M), f"{kernel}: {fname} has no {test}"
        assert re.search(rf"^ *\d+ {re.escape(kernel)}$", trace, flags=re.M), kernel
