"""The division of the paged attention's workspace, compiled for the host: whatever its words hold where a wait of the first kernel ran
out, the second one follows no span of pieces out of the workspace."""
import ctypes as C
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")
SMS = 148

SOURCE = """
#include "paged_plan.cuh"
using namespace mtv;
extern "C" long long plan(int sms, int T, int B, int G, int Hkv, int D, int shared, long long *out) {
    PaPhase ph[3];
    char *base = reinterpret_cast<char *>(1 << 20);
    const size_t bytes = pa_plan(ph, sms, T, B, G, Hkv, D, shared, base);
    for (int f = 0; f < 3; ++f) {
        const long long v[7] = {ph[f].prefix_items + (long long)B * ph[f].seq_items, ph[f].rows, ph[f].workers,
                                reinterpret_cast<char *>(ph[f].o) - base, reinterpret_cast<char *>(ph[f].ml) - base,
                                reinterpret_cast<char *>(ph[f].span) - base, 0};
        for (int i = 0; i < 7; ++i) out[f * 7 + i] = v[i];
    }
    return (long long)bytes;
}
extern "C" int span_ok(int workers, int x, int y) {
    PaPhase f = {};
    f.workers = workers;
    return pa_span_ok(f, make_int2(x, y));
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, lib = d / "plan.cpp", d / "plan.so"
    src.write_text(SOURCE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-I", os.path.join(ROOT, "paper_2603_03383_b200", "csrc"), "-I",
                           os.path.join(CUDA, "include"), "-o", str(lib), str(src)])
    L = C.CDLL(str(lib))
    L.plan.restype = C.c_longlong
    return L


@pytest.mark.parametrize("T,B,G,Hkv,D,shared", [
    (1, 1, 4, 1, 128, 0), (1, 64, 4, 8, 128, 8192), (29, 7, 7, 4, 128, 1008), (128, 3, 8, 2, 64, 4096), (64, 8, 4, 8, 128, 16384), (4, 2, 4, 1, 64, 16),
    (1, 1024, 2, 1, 64, 32), (65, 2, 6, 1, 64, 384),
])
def test_no_span_leads_out_of_the_workspace(host, T, B, G, Hkv, D, shared):
    out = (C.c_longlong * 21)()
    total = host.plan(SMS, T, B, G, Hkv, D, shared, out)
    words = [-2 ** 31, -1, 0, 1, 2, SMS - 1, SMS, 2 * SMS - 1, 2 * SMS, 2 * SMS + 1, 0x7f7f7f7f, 2 ** 31 - 1]
    words += torch.randint(-2 ** 31, 2 ** 31, (20,), generator=torch.Generator().manual_seed(1)).tolist()
    phases = [out[f * 7:f * 7 + 6] for f in range(3)]
    starts = sorted([x for ph in phases for x in ph[3:6]] + [total])
    followed = 0
    for items, rows, workers, o, ml, span in phases:
        end = lambda x: min(s for s in starts if s > x)  # noqa: E731
        if items == 0:
            assert workers == 0 and not any(host.span_ok(workers, x, y) for x in words for y in words)
            continue
        assert span + 8 * items <= end(span)
        for x in words:
            for y in words:
                if host.span_ok(workers, x, y):
                    followed += 1
                    for item in (0, items - 1):
                        assert item + x >= 0 and y - x + 1 >= 1
                        assert o + (item + y + 1) * rows * D * 4 <= end(o) and ml + (item + y + 1) * rows * 8 <= end(ml)
        # what the first kernel writes passes: any run of workers
        assert host.span_ok(workers, 0, 0) and host.span_ok(workers, 0, workers - 1) and host.span_ok(workers, workers - 1, workers - 1)
    assert followed


def test_the_joining_kernel_asks():
    """Both spans of a row are looked at before either becomes an address."""
    text = open(os.path.join(ROOT, "paper_2603_03383_b200", "csrc", "attention_paged.cu")).read()
    kernel = text[text.index("paged_attn_combine_kernel(const"):]
    asked, used = kernel.index("(!p.shared || pa_span_ok(f0, span0)) && pa_span_ok(f1, span1)"), kernel.index("s1 = source(")
    assert asked < used
