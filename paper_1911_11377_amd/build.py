"""Build the HIP library (libckksmi.so, gfx950) in-tree with hipcc."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libckksmi.so")
SOURCES = ["ckksmi_device.hip", "train_device.hip", "norm_device.hip", "muon_device.hip", "low_device.hip", "host_math.cpp", "host_crypto.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off",
    # keep the compiler from forming packed-FP32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unknown-attributes",
]


def build(force=True):
    srcs = [os.path.join(CSRC, s) for s in SOURCES]
    deps = srcs + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h")]
    deps += [os.path.join(HERE, "..", "include", h) for h in ("ckksmi.h", "ckksmi_profile.h", "ckksmi_train.h")]
    if not force and os.path.exists(LIB) and all(os.path.getmtime(LIB) >= os.path.getmtime(d) for d in deps):
        return LIB
    tmp = LIB + ".tmp.%d" % os.getpid()
    objects = ["%s.%d.o" % (tmp, i) for i in range(len(srcs))]
    compile_flags = [f for f in FLAGS if f != "-shared"]
    try:
        # the device sources take up to minutes: side by side
        running = [subprocess.Popen([HIPCC] + compile_flags + ["-c", "-x", "hip", s, "-o", o]) for s, o in zip(srcs, objects)]
        failed = [s for s, p in zip(srcs, running) if p.wait() != 0]
        if failed:
            raise RuntimeError("compilation failed: %s" % ", ".join(failed))
        subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC"] + objects + ["-o", tmp])
        os.replace(tmp, LIB)
    finally:
        for f in objects:
            if os.path.exists(f):
                os.remove(f)
    return LIB


if __name__ == "__main__":
    print(build())
