"""What the compiler made of the latent-cache and page kernels, the headers as C99, and their host code under sanitizers (no GPU)."""
import ctypes
import os
import re
import subprocess
import sys

import pytest

from paper_2605_06914_amd.build import CSRC, HIP_FLAGS, ROOT
from tests.asm_hazards import scan, scan_scalar_addresses

SOURCES = {"taper_latent_kernels.hip": 13, "taper_prompt_kernels.hip": 8, "taper_pages_kernels.hip": 6}


@pytest.fixture(scope="module", params=SOURCES, ids=lambda s: s.split(".")[0])
def compiled(request, tmp_path_factory):
    asm = tmp_path_factory.mktemp("kernels") / "kernels.s"
    flags = [f for f in HIP_FLAGS if f not in ("-shared", "-fPIC")]
    cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "--cuda-device-only", "-S", "-Rpass-analysis=kernel-resource-usage",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", str(asm), os.path.join(CSRC, request.param)]
    run = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
    assert run.returncode == 0, run.stderr[-2000:]
    return request.param, asm.read_text(), run.stderr


def test_kernels_use_no_scratch_memory_and_nothing_is_warned_of(compiled):
    source, _, remarks = compiled
    found = re.findall(r"Function Name: (\S+)(?:.|\n)*?ScratchSize \[bytes/lane\]: (\d+)", remarks)
    assert len(found) == SOURCES[source], found
    assert all(n == "0" for _, n in found), found
    assert [l for l in remarks.splitlines() if "warning:" in l] == []


def test_no_matrix_result_and_no_scalar_address_is_read_too_early(compiled):
    source, asm, _ = compiled
    for check in (scan, scan_scalar_addresses):
        findings, kernels = check(asm, name_filter="kernel")
        assert kernels == SOURCES[source] and not findings, findings[:5]


def test_ctypes_structures_mirror_the_headers_and_the_headers_are_c99(tmp_path):
    from paper_2605_06914_amd import latent, pages
    classes = [latent.taper_latent_config, latent.taper_latent_item, latent.taper_latent_view, pages.taper_page_format]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "taper_latent.h"', '#include "taper_pages.h"', "int main(void) {"]
    for c in classes:
        n = c.__name__
        lines.append(f'    printf("{n} %zu\\n", sizeof({n}));')
        lines += [f'    printf("{n}.{f} %zu %zu\\n", offsetof({n}, {f}), sizeof((({n} *)0)->{f}));' for f, _ in c._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["    return 0;", "}"]) + "\n")
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    seen = {k: tuple(map(int, v)) for k, *v in (l.split() for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())}
    for c in classes:
        assert seen[c.__name__] == (ctypes.sizeof(c),)
        for f, _ in c._fields_:
            assert seen[f"{c.__name__}.{f}"] == (getattr(c, f).offset, getattr(c, f).size)


STUBS = """
#include "latent_kernels.h"
#include "pages_kernels.h"
namespace taper {
hipError_t launch_latent_decode(const LatentShape&, const LatentDecodeArgs&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_latent_prompt(const LatentShape&, const PromptArgs&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_latent_append(int, int64_t, const void*, int64_t, const void*, int64_t, const int64_t*, void*, int64_t, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_pages_copy(const PoolPointers&, int, const PageMove*, const MoveArguments*, int64_t, int64_t, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_pages_pack(const PoolPointers&, int, const PackArgs&, hipStream_t) { return hipErrorNotSupported; }
}
"""


def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    asan = subprocess.run(["gcc", "-print-file-name=libasan.so"], capture_output=True, text=True).stdout.strip()
    if not os.path.isabs(asan) or not os.path.exists(asan):
        pytest.skip("no libasan.so beside gcc")
    (tmp_path / "stubs.cpp").write_text(STUBS)
    lib = tmp_path / "libtaper_attn_san.so"
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer", "-g", "-O1"]
    subprocess.check_call(["g++", "-std=c++17", "-fPIC", "-shared", *san, "-D__HIP_PLATFORM_AMD__", "-fvisibility=hidden", "-I", os.path.join(ROOT, "include"),
                           "-I", CSRC, "-I", "/opt/rocm/include", "-o", str(lib), *[os.path.join(CSRC, f) for f in (
                               "taper_api.cpp", "taper_plan.cpp", "taper_admission.cpp", "taper_latent.cpp", "taper_pages.cpp")],
                           str(tmp_path / "stubs.cpp"), os.path.join(ROOT, "tests", "sanitize", "kernel_stubs.cpp"),
                           "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"])
    code = (f"import sys; sys.path.insert(0, {ROOT!r})\nfrom paper_2605_06914_amd import binding\nbinding.LIB_PATH = {str(lib)!r}\nimport pytest\n"
            f"sys.exit(pytest.main(['-q', '-x', '-p', 'no:cacheprovider', {os.path.join(ROOT, 'tests', 'test_latent_host.py')!r}, "
            f"{os.path.join(ROOT, 'tests', 'test_pages_host.py')!r}]))")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1",
               LD_PRELOAD=asan + (":" + os.environ["LD_PRELOAD"] if os.environ.get("LD_PRELOAD") else ""))
    run = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True, timeout=1500, cwd=ROOT)
    out = run.stdout + run.stderr
    assert "AddressSanitizer" not in out and "runtime error:" not in out and run.returncode == 0 and " passed" in run.stdout, out[-4000:]
