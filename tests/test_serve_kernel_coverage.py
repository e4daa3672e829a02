"""Every kernel instantiation compiled into libsparrow_serve.so and the GPU test that runs it against the formulas: the keys must be exactly the
`__global__` instantiations the library holds, and every test named must exist.  That each runs in the GPU tests of the serving operators was observed
with a kernel trace (profiles/serve_gpu_test_kernel_coverage.txt)."""
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2602_15318_amd", "libsparrow_serve.so")

C8, AT, RA = "test_gpu_serve_cache8.py", "test_gpu_serve_attn.py", "test_gpu_serve_ranges.py"
BF16, F32, E4M3 = "unsigned short", "float", "unsigned char"
COVERAGE = {
    **{f"mrope_append8_kernel<{t}, {d}>": (C8, "test_append") for t in (F32, BF16) for d in (64, 128)},
    # <storage type of the output, of the cache, head_dim>
    **{f"page_gather_kernel<{t}, {c}, {d}>": (C8, "test_gather") for t in (F32, BF16) for c in (t, E4M3) for d in (64, 128)},
    "serve_plan_kernel": (AT, "test_shared_prefixes"),
    # more than 16 rows (new token, query head of the group) per KV head, or groups
    **{f"serve_attn_kernel<{c}, {d}>": (AT, "test_shared_prefixes") for c in (BF16, E4M3) for d in (64, 128)},
    **{f"serve_attn_f32_kernel<{c}, {d}>": (AT, "test_shared_prefixes") for c in (F32, E4M3) for d in (64, 128)},
    # <storage type of the cache, head_dim, wavefronts>: up to 16 rows
    **{f"serve_few_kernel<{c}, 64, {w}>": (RA, "test_batches_of_every_size") for c in (BF16, E4M3) for w in (2, 4, 8)},
    **{f"serve_few_kernel<{c}, 128, {w}>": (RA, "test_batches_of_heads_of_128") for c in (BF16, E4M3) for w in (2, 4)},
    **{f"serve_few_kernel<{c}, 128, 8>": (RA, "test_long_contexts") for c in (BF16, E4M3)},
    # 17 to 64 rows a request at most
    **{f"serve_some_kernel<{c}, {d}>": (AT, "test_chains") for c in (BF16, E4M3) for d in (64, 128)},
    # <storage type, head_dim, wavefronts that share a row's pieces>
    **{f"serve_combine_kernel<{t}, {d}, {n}>": (AT, "test_shared_prefixes") for t in (F32, BF16) for d in (64, 128) for n in (1, 2, 8)},
}


def test_every_compiled_kernel_instantiation_has_a_test():
    if not os.path.exists(LIB):
        from paper_2602_15318_amd import build
        build.build()
    out = subprocess.run(["nm", "-C", LIB], capture_output=True, text=True, check=True).stdout
    compiled = set(re.sub(r".*::", "", k) for k in re.findall(r"__device_stub__(.*?)\(", out))
    assert compiled == set(COVERAGE), (sorted(compiled - set(COVERAGE)), sorted(set(COVERAGE) - compiled))


def test_the_named_tests_exist_and_the_trace_has_them():
    trace = open(os.path.join(ROOT, "profiles", "serve_gpu_test_kernel_coverage.txt")).read()
    for kernel, (fname, test) in COVERAGE.items():
        src = open(os.path.join(ROOT, "tests", fname)).read()
        assert re.search(rf"^def {test}\(", src, flags=re.M), f"{kernel}: {fname} has no {test}"
        assert re.search(rf"^ *\d+ {re.escape(kernel)}$", trace, flags=re.M), kernel
