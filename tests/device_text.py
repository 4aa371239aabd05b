"""Runs device functions of the kernels' sources on the CPU: takes their text out of the files and compiles it as C++."""
import ctypes
import hashlib
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2110_04175_gb300", "csrc")

SHIM = """
#include <cmath>
#include <cstdint>
#include <cstring>
#define __device__
#define __forceinline__ inline
struct float2 { float x, y; };
static inline float2 make_float2(float x, float y) { return {x, y}; }
static inline uint32_t __float_as_uint(float f) { uint32_t u; std::memcpy(&u, &f, 4); return u; }
static inline float __uint_as_float(uint32_t u) { float f; std::memcpy(&f, &u, 4); return f; }
static inline float __int_as_float(int32_t u) { return __uint_as_float(static_cast<uint32_t>(u)); }
"""


def text_of(source, name):
    """Every definition of the function or struct `name` in the file, templates' heads included."""
    text = open(os.path.join(CSRC, source)).read()
    found = []
    for at in re.finditer(r"^(?:template <[^\n]*>\n)?(?:struct %s \{|__device__ __forceinline__ [^\n(]*\b%s\()" % (name, name), text, re.M):
        depth, i = 0, text.index("{", at.end() - 1)
        while True:
            depth += {"{": 1, "}": -1}.get(text[i], 0)
            i += 1
            if depth == 0:
                break
        found.append(text[at.start():i] + (";" if "struct" in at.group().split("\n")[-1][:6] else ""))
    assert found, f"{name} is not in {source}"
    return "\n".join(found)


def compiled(folder, parts, body):
    """A library of `body` (C++, extern "C") behind the named functions [(source, name)]."""
    code = SHIM + "\n".join(part if isinstance(part, str) else text_of(*part) for part in parts) + '\nextern "C" {\n' + body + "\n}\n"
    path = os.path.join(str(folder), "device_" + hashlib.sha1(code.encode()).hexdigest()[:12])
    with open(path + ".cpp", "w") as f:
        f.write(code)
    subprocess.run(["g++", "-std=c++17", "-O1", "-ffp-contract=off", "-Wno-unknown-pragmas", "-shared", "-fPIC", path + ".cpp", "-o",
                    path + ".so"], check=True)
    return ctypes.CDLL(path + ".so")
