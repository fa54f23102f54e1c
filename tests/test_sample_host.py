"""The sampling's workgroup with checked memory, on the host: csrc/sample.h, its storage replaced by cells with bounds, writers and readers (sample_host.cpp),
over rows that take each of its ways.  No index leaves its array, no load its row, nothing is read that was not written, nothing is raced for, and
the tokens are the oracle's."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from test_gpu_lm import check_tokens

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_11168_amd", "csrc")


def _replace(text, old, new, count=1):
    assert text.count(old) == count, (old, text.count(old))
    return text.replace(old, new)


def _cells(text, name):
    """The members of struct `name` as cells."""
    begin = text.index("struct %s {" % name)
    end = text.index("};", begin)
    body = re.sub(r"//[^\n]*", "", text[begin:end])
    head, members = body.split("{", 1)
    out = []
    for line in filter(None, (m.strip() for m in members.split(";"))):
        kind, names = line.split(" ", 1)
        for n in names.split(","):
            array = re.fullmatch(r"\s*(\w+)\[(.+)\]", n)
            out.append("  emu::Array<%s, %s> %s;" % (kind, array[2], array[1]) if array else "  emu::Cell<%s> %s;" % (kind, n.strip()))
    return text[:begin] + head + "{\n" + "\n".join(out) + "\n" + text[end:]


def _sources(to, plant=None):
    rows = open(os.path.join(CSRC, "rows.h")).read()
    rows = re.sub(r'#include [<"].*\n', "", rows)
    rows = rows[:rows.index("// Values of other lanes")] + "}  // namespace elmo\n"
    for kind in ("uint16_t", "float"):
        rows = re.sub(r"(load_octet\(const %s\* __restrict__ p, int64_t valid, %s fill = [\w.]+\) \{\n)" % (kind, kind),
                      r"\1  emu::global(p, (valid < 8 ? valid : 8) * sizeof *p);\n", rows)
        rows = _replace(rows, "load_one<%s>(const %s* p, int64_t i) { return" % (kind, kind), "load_one<%s>(const %s* p, int64_t i) { emu::global(p + i, sizeof *p); return" % (kind, kind))
    assert rows.count("emu::global") == 4
    (to / "host_rows.h").write_text(rows)
    text = open(os.path.join(CSRC, "sample.h")).read()
    text = _replace(text, '#include "rows.h"\n', "")
    for name in ("SampleLds", "SampleWs", "SampleCodes"):
        text = _cells(text, name)
    text = text[:text.index("enum : int { SAMPLE_WHOLE")] + "}  // namespace elmo\n"
    text = _replace(text, "U* slots", "typename emu::Same<emu::Ptr<U>>::type slots")
    text = _replace(text, "sort_falling(uint64_t* s", "sort_falling(emu::Ptr<uint64_t> s")
    text = _replace(text, "rank_falling(uint64_t* list, uint32_t* rank", "rank_falling(emu::Ptr<uint64_t> list, emu::Ptr<uint32_t> rank")
    text = _replace(text, "const double* roots;", "emu::Ptr<double> roots;")
    text = _replace(text, "n0 = l.count[2 * tid], n1 = l.count[2 * tid + 1];", "n0 = l.count[2 * tid] + 0, n1 = l.count[2 * tid + 1] + 0;")
    text = text.replace("(unsigned long long*)&", "&")
    (to / "host_sample.h").write_text(_replace(text, *plant) if plant else text)


def _build(d, plant=None):
    _sources(d, plant)
    lib = str(d / "sample_host.so")
    subprocess.run([os.environ.get("HOSTCXX", "/opt/rocm/llvm/bin/clang++"), "-std=c++17", "-O1", "-ffp-contract=off", "-Wno-deprecated", "-shared", "-fPIC",
                    "-I", str(d), "-o", lib, os.path.join(ROOT, "tests", "sample_host.cpp")], check=True)
    f = ctypes.CDLL(lib).host_sample
    P, L = ctypes.c_void_p, ctypes.c_int64
    f.restype, f.argtypes = ctypes.c_char_p, [P, L, ctypes.c_int, L, L, P, P, P, P, P, P, P, ctypes.c_int]

    def sample(z, u, parts=1, t=None, top_k=None, top_p=None, min_p=None):
        token, prob = torch.full((len(u),), -7, dtype=torch.int32), torch.full((len(u),), -7.0)
        p = lambda v: None if v is None else v.data_ptr()  # noqa: E731
        said = f(z.data_ptr(), z.stride(0), int(z.dtype == torch.float32), z.shape[0], z.shape[1], p(u), p(t), p(top_k), p(top_p), p(min_p), p(token), p(prob), parts)
        assert said is None, said.decode()
        return token, prob
    return sample


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    return _build(tmp_path_factory.mktemp("sample_host"))


def odd_rows(rows, V, dtype, g):
    """Ordinary rows; among the first of them empty ones, ones of infinities, zeros, one value, values next to zero, far from it and over the whole type."""
    z = 2.5 * torch.randn((rows, V), generator=g)
    z[0, V // 2:] = -float("inf")
    z[1, V // 3], z[1, V - 1] = float("inf"), float("inf")
    z[2] = torch.where(torch.rand(V, generator=g) < 0.3, 0.0, z[2])
    z[3] = -float("inf")
    z[4] = -3.0
    z[5] *= 1e-6
    z[6] = 1000 + 8 * torch.randn(V, generator=g)
    z[7] *= 4e36
    z[8] = -z[2].abs()
    z[9, ::2] = float("nan")
    return z.to(dtype)


SETTINGS = [dict(), dict(top_p=0.9), dict(top_p=0.3, t=0.7), dict(min_p=0.05), dict(top_p=0.97, min_p=0.01, t=1.5), dict(t=0.0), dict(top_p=0.5, t=1e30), dict(top_p=0.8, t=1e-3),
            dict(top_k=1), dict(top_k=40, top_p=0.9), dict(top_k=400, min_p=0.01), dict(top_k=700, top_p=0.8), dict(t=float("inf")), dict(min_p=1.0)]


def settings(rows, kw):
    return {n: torch.full((rows,), v, dtype=torch.int32 if n == "top_k" else torch.float32) for n, v in kw.items()}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,parts", [(1, 1), (5, 1), (700, 1), (20011, 1), (20011, 2), (65543, 16)])
def test_a_workgroup_stays_in_its_memory(host, V, parts, dtype):
    g = torch.Generator()
    g.manual_seed(V)
    rows = 11
    z = odd_rows(rows, V, dtype, g)
    for kw in SETTINGS:
        if parts > 1 and "top_k" in kw:
            continue                                         # (never split)
        u, s = torch.rand(rows, generator=g), settings(rows, kw)
        token, prob = host(z, u, parts, **s)
        if kw.get("t") == float("inf"):                      # all alike
            s["t"] = torch.full((rows,), 1e300, dtype=torch.float64)
        check_tokens(z, u, token, prob, **s)
        if parts > 1:
            whole, prob1 = host(z, u, 1, **settings(rows, kw))
            assert torch.equal(whole, token) and torch.equal(prob1, prob)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ties_of_thousands(host, dtype):
    """Lists that overflow, a filter's end among more equal logits than a list holds, a list of full length."""
    g = torch.Generator()
    g.manual_seed(1)
    V = 20011
    z = torch.randint(0, 3, (5, V), generator=g).to(dtype)
    z[0] = 1.0
    z[1] = (8 * torch.rand(V, generator=g)).round().to(dtype) / 8       # some 2500 equal ones
    z[2] = torch.where(torch.arange(V) % 5 == 0, z[2].float(), -40.0).to(dtype)
    for kw in (dict(), dict(top_k=V // 2 + 1), dict(top_p=0.7), dict(top_k=V // 3, top_p=0.5), dict(min_p=0.2), dict(top_k=1000), dict(top_k=500, top_p=0.6), dict(top_p=0.7, t=1e-3)):
        u, s = torch.rand(5, generator=g), settings(5, kw)
        for parts in (1, 4):
            if parts == 1 or "top_k" not in kw:
                token, prob = host(z, u, parts, **s)
                check_tokens(z, u, token, prob, **s)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_segments_of_several_rounds(host, dtype):
    """Above 2097152 tokens."""
    g = torch.Generator()
    g.manual_seed(2)
    V = 2_200_003
    z = (2.5 * torch.randn((1, V), generator=g)).to(dtype)
    for kw in (dict(), dict(top_p=0.9), dict(top_k=50), dict(top_k=1000, top_p=0.8), dict(t=0.0)):
        u, s = torch.rand(1, generator=g), settings(1, kw)
        for parts in (1, 7):
            if parts == 1 or "top_k" not in kw:
                token, prob = host(z, u, parts, **s)
                check_tokens(z, u, token, prob, **s)


@pytest.mark.parametrize("plant,said", [
    (("if (tid < 3) l.found[tid] = tid == 0 ? kNoEnd : 0;", "if (tid == 0) l.found[0] = kNoEnd;"), "nobody wrote"),
    (("  if (tid < kSampleCount) rank[tid] = 0;\n  __syncthreads();\n", "  if (tid < kSampleCount) rank[tid] = 0;\n"), "same interval"),
    (("min(-n >> 2, kSampleBins - 1)", "min(-n >> 2, kSampleBins)"), "outside its array"),
    (("load_octet(z + o * 8, a.V - o * 8, lowest<T>())", "load_octet(z + o * 8, 8, lowest<T>())"), "outside the row")])
def test_the_checks_find_planted_mistakes(tmp_path, plant, said):
    planted = _build(tmp_path, plant)
    g = torch.Generator()
    g.manual_seed(3)
    V = 20011
    with pytest.raises(AssertionError, match=said):
        for dtype in (torch.bfloat16, torch.float32):
            z = odd_rows(10, V, dtype, g)
            z[:, 5] = -30.0                                  # a weight behind the last bin
            for kw in (dict(top_p=0.9), dict(top_k=40)):
                planted(z, torch.rand(10, generator=g), **settings(10, kw))


def test_the_kernels_neither_call_nor_use_scratch(tmp_path):
    """Sampler is one body of instructions, LDS reached as LDS: no call, no stack, no flat access (nor in any other of the output end's kernels)."""
    from paper_2510_11168_amd import build
    if not build.is_built():
        build.build()
    shutil.copy(build.LIB_PATH, tmp_path / "lib.so")
    llvm = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")
    subprocess.run([os.path.join(llvm, "llvm-objdump"), "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    seen = 0
    for f in sorted(tmp_path.glob("lib.so.*gfx950")):
        notes = subprocess.run([os.path.join(llvm, "llvm-readelf"), "--notes", str(f)], check=True, capture_output=True, text=True).stdout
        if "k_sample" not in notes:
            continue
        sizes = re.findall(r"\.private_segment_fixed_size: *(\d+)", notes)
        seen += notes.count("k_sample")
        assert sizes and set(sizes) == {"0"}
        code = subprocess.run([os.path.join(llvm, "llvm-objdump"), "-d", "--no-show-raw-insn", str(f)], check=True, capture_output=True, text=True).stdout
        assert not re.search(r"\t(s_swappc|flat_|scratch_)\w+", code)
    assert seen
