"""Build libgorgo.so (HIP, gfx950 only) in-tree with hipcc.  Every call compiles: the sources include every header
under csrc/, and nothing here guesses whether an existing library is still current."""
import os
import re
import shutil
import struct
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libgorgo.so")
SOURCES = ["trace.cpp", "es.cpp", "api.cpp", "kernels.hip"]
# (a compilation of its own: the scheduling strategy that suits the replay kernels' chains costs these registers)
ATTENTION_SOURCES = ["attention.cpp", "attention.hip", "append.cpp", "append.hip"]


def _run(cmds, verbose: bool) -> None:
    """Runs the commands side by side."""
    if verbose:
        for cmd in cmds:
            print(" ".join(cmd))
    running = [subprocess.Popen(cmd, stderr=subprocess.PIPE, text=True) for cmd in cmds]
    failed = False
    for p in running:
        err = p.communicate()[1]
        # the host pass does not know the device-only target feature and says so once per file: harmless
        noise = "'-packed-fp32-ops' is not a recognized feature"
        err = "\n".join(l for l in err.splitlines() if noise not in l)
        if err.strip():
            print(err)
        failed = failed or p.returncode != 0
    if failed:
        raise RuntimeError("hipcc failed")


def _code_objects(path: str):
    """The GPU's ELF files in a library."""
    data = open(path, "rb").read()
    at = data.find(b"\x7fELF", 4)
    while at >= 0:
        if struct.unpack_from("<H", data, at + 18)[0] == 224:                  # AMDGPU
            sections, = struct.unpack_from("<Q", data, at + 40)
            size, count = struct.unpack_from("<HH", data, at + 58)
            yield data[at:at + sections + size * count]
        at = data.find(b"\x7fELF", at + 4)


def _kernels(elf: bytes) -> dict:
    """Of each kernel, by its descriptor: vector registers that a wavefront is given, and bytes of scratch memory a lane."""
    table, = struct.unpack_from("<Q", elf, 40)
    size, count = struct.unpack_from("<HH", elf, 58)
    sections = [struct.unpack_from("<IIQQQQIIQQ", elf, table + i * size) for i in range(count)]
    out = {}
    for _, kind, _, _, offset, length, link, _, _, entry in sections:
        if kind != 2:                                                           # symbols
            continue
        for symbol in range(offset, offset + length, entry):
            name, _, _, section, value, _ = struct.unpack_from("<IBBHQQ", elf, symbol)
            begin = sections[link][4] + name
            text = elf[begin:elf.index(b"\0", begin)].decode()
            if text.endswith(".kd"):
                descriptor = sections[section][4] + value - sections[section][3]
                scratch, registers = (struct.unpack_from("<I", elf, descriptor + at)[0] for at in (4, 48))
                out[text[:-3]] = ((registers & 63) + 1) * 8, scratch
    return out


def shifts_by_the_last_register(path: str, hipcc: str = "/opt/rocm/bin/hipcc") -> list:
    """64-bit shifts whose amount lies in the last vector register that a wavefront is given, as (kernel, instruction).  On gfx950 such a shift now and
    then shifts by nothing (a quarter of them where four wavefronts of 128 registers fill a SIMD, none where one workgroup runs alone), and the
    compiler does not avoid it.  Of instructions that read 32 bits beside 64 the three shifts are the ones it happens to; sums after a shift,
    products, conversions and powers of two of doubles are as they should be (4e9 of each compared)."""
    objdump = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(shutil.which(hipcc) or hipcc))), "llvm", "bin", "llvm-objdump")
    found = []
    for elf in _code_objects(path):
        kernels = _kernels(elf)
        with tempfile.NamedTemporaryFile(suffix=".co") as f:
            f.write(elf)
            f.flush()
            listing = subprocess.run([objdump, "-d", "--no-show-raw-insn", "--mcpu=gfx950", f.name], check=True, capture_output=True, text=True).stdout
        for line in listing.splitlines():
            label = re.match(r"[0-9a-f]+ <(.+)>:$", line)
            if label:
                name, given = label[1], kernels.get(label[1], (None,))[0]
            shift = re.match(r"\s+((?:v_lshlrev_b64|v_lshrrev_b64|v_ashrrev_i64)\S*\s+v\[\d+:\d+\], v(\d+), .*?)\s*(?://.*)?$", line)
            # (a function that is no kernel runs with any caller's registers)
            if shift and (int(shift[2]) == given - 1 if given else int(shift[2]) % 8 == 7):
                found.append((name, shift[1]))
    return found


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    common = [hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
              # every fp64 product and sum on the decision path is rounded on its own: no fused multiply-add
              "-ffp-contract=off", "-fno-fast-math",
              "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
              "-Wall", "-Wno-unused-command-line-argument",
              "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    # the replay kernels are long dependent chains: scheduling for instruction-level parallelism measures
    # about 2 % faster than the default (occupancy-first) strategy
    replay = ["-mllvm", "-amdgpu-sched-strategy=max-ilp"]
    with tempfile.TemporaryDirectory() as tmp:
        objects, cmds = [], []
        for flags, sources in ((replay, SOURCES), ([], ATTENTION_SOURCES)):
            for src in sources:
                objects.append(os.path.join(tmp, src + ".o"))
                cmds.append(common + flags + ["-x", "hip", "-c", os.path.join(CSRC, src), "-o", objects[-1]])
        _run(cmds, verbose)
        _run([[hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + objects + ["-o", LIB]], verbose)
    shifts = shifts_by_the_last_register(LIB, hipcc)
    if shifts:
        raise RuntimeError(f"64-bit shifts by a wavefront's last register, which gfx950 does not always do: {shifts}")
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
