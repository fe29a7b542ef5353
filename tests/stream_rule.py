"""The rules by which the streaming attention cuts sequences (csrc/stream_cut.h), compiled by themselves."""
import ctypes as C
import functools
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_19602_b200", "csrc")
SMS = 148
CODE = """#include "stream_cut.h"
using namespace scalekv::paged;
extern "C" int ctas(int d, int q8, int n) { return stream_ctas(d, q8, n); }
extern "C" void cut(int n_sm, int slots, int n_seqs, long long items, long long rows, long long keys, int *out) {
  const StreamCut c = cut_stream(n_sm, slots, n_seqs, items, rows, keys);
  out[0] = c.split; out[1] = c.most_parts;
}
extern "C" void deal(long long total, int longest, int items, int ctas, int most_parts, int *out) {
  const StreamDeal d = deal_steps(total, longest, items, ctas, most_parts);
  out[0] = d.split; out[1] = d.share;
}
extern "C" long long part_rows() { return kPartRows; }
extern "C" int max_counts() { return kMaxCounts; }
extern "C" int most() { return kMostParts; }
"""


@functools.lru_cache(None)
def library():
    with tempfile.TemporaryDirectory() as at:
        with open(os.path.join(at, "rule.cpp"), "w") as f:
            f.write(CODE)
        subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I", CSRC, os.path.join(at, "rule.cpp"), "-o", os.path.join(at, "rule.so")], check=True)
        lib = C.CDLL(os.path.join(at, "rule.so"))
    lib.part_rows.restype = C.c_longlong
    return lib


def slots(d, store, rows, n_sm=SMS):
    """CTAs that the device has room for, with `rows` query rows to a sequence and kv head."""
    return n_sm * library().ctas(d, int(store == "q8"), 1 if rows <= 8 else 2)


def cut(slots, n_seqs, items, rows, keys, n_sm=SMS):
    """(CTAs that share a sequence's keys, most parts of a sequence and head where they are dealt out by the lengths)"""
    out = (C.c_int * 2)()
    library().cut(n_sm, slots, n_seqs, C.c_longlong(items), C.c_longlong(rows), C.c_longlong(keys), out)
    return out[0], out[1]


def deal(total, longest, items, ctas, most_parts):
    """(equal parts of a sequence and head, steps of a CTA where all steps are shared out evenly or 0)"""
    out = (C.c_int * 2)()
    library().deal(C.c_longlong(total), longest, items, ctas, most_parts, out)
    return out[0], out[1]
