"""The plan of a pc_shared_attn call is arithmetic on the host over whatever sizes the checks let through: built for the CPU
alone with the compiler's check for signed overflow, no size ends the program."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC, INCLUDE = os.path.join(ROOT, "paper_2502_14317_amd", "csrc"), os.path.join(ROOT, "include")


def test_no_overflow(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    checked = ["-Xarch_host", "-fsanitize=signed-integer-overflow", "-Xarch_host", "-fno-sanitize-recover=signed-integer-overflow"]
    common = ["--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-Wno-unused-command-line-argument", "-I", INCLUDE, "-I", CSRC]
    objects, running = [], []
    for name in ("shared_attn", "serve_api", "pc_api", "row8", "verify"):
        objects.append(str(tmp_path / f"{name}.o"))
        running.append(subprocess.Popen([hipcc, *common, *checked, "-c", os.path.join(CSRC, f"{name}.hip"), "-o", objects[-1]],
                                        stderr=subprocess.PIPE, text=True))
    for p in running:
        assert p.wait() == 0, p.stderr.read()
    # kernels and the other files' functions are never called
    program = str(tmp_path / "check")
    subprocess.run(["/opt/rocm/llvm/bin/clang++", "-std=c++17", "-fsanitize=signed-integer-overflow", "-I", INCLUDE,
                    os.path.join(ROOT, "tests", "host", "shared_plan_check.cpp"), *objects, "-o", program, "-L/opt/rocm/lib", "-lamdhip64",
                    "-Wl,--unresolved-symbols=ignore-all", "-Wl,-rpath,/opt/rocm/lib"], check=True, capture_output=True)
    r = subprocess.run([program], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert int(r.stdout) > 1000
