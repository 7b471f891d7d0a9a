"""CPU: the descriptor tables that kernels get as arguments are aligned for what the kernels read in them (csrc/call_tables.h), wherever they
stand among the arguments."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include "attend_few.h"
#include "attend_selected.h"
#include "block_select.h"
#include "kv_move.h"
#include "rope_append.h"
template <class Tab, class... Reqs>
constexpr bool aligned_for() { return ((alignof(Tab) % alignof(Reqs) == 0) && ...) && sizeof(Tab) % 16 == 0; }
template <class Tab>
constexpr bool good() { return aligned_for<Tab, PageCopy, MoveReq, FewReq, FewShared, BoundsReq, BoundsAt, SelectReq, AppendItem, uint4>(); }
static_assert(good<InlineTable>(), "InlineTable");
static_assert(good<SmallTable>(), "SmallTable");
static_assert(alignof(PageCopy) == 8 && alignof(MoveReq) == 8, "64-bit addresses");
struct Arguments { int hkv; InlineTable tab; };   // page_copy_kernel's
static_assert(offsetof(Arguments, tab) % alignof(PageCopy) == 0, "behind an int");
"""


def test_tables_are_aligned_for_their_requests(tmp_path):
    from paper_2509_24381_amd.build import HIPCC_FLAGS
    src = tmp_path / "tables.hip"
    src.write_text(SOURCE)
    flags = [f for f in HIPCC_FLAGS if f not in ("-shared", "-fPIC", "-O3")]
    r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "-I", os.path.join(ROOT, "paper_2509_24381_amd", "csrc"), "-fsyntax-only", str(src)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
