"""The launches that attention over pages makes of a batch's sizes (csrc/paged_plan.h), checked on
the CPU: every form that a batch can take is one of FORMS, which the GPU tests run."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HARNESS = r"""
#include <cstdio>
#include <cstdlib>
#include "paged_plan.h"

// lines of: heads kv_heads head_dim n_seq rows max_rows max_len
int main() {
  int a[7];
  while (scanf("%d %d %d %d %d %d %d", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6) == 7) {
    const PagedPlan p = paged_attention_plan(a[0], a[1], a[2], a[3], a[4], a[5], a[6]);
    printf("%d %lld", p.fits, (long long)p.bytes);
    for (int i = 0; i < p.n; ++i)
      printf(" %d %d %lld %d %d", p.part[i].wm, p.part[i].single, (long long)p.part[i].slots, p.part[i].splits,
             p.part[i].chunk);
    puts("");
  }
  return 0;
}
"""

# (new rows, tokens with them) of each sequence, query heads, K / V heads, head_dim; the row tiles of
# each launch: 32 rows x this, one tile a sequence at most, key splits (1: whole, 2: 2 to 16, 3: more)
FORMS = {
    "32 rows": ([(1, 700)] * 64, 8, 8, 128, [(1, 1, 1)]),
    "32 rows, d 64": ([(1, 700)] * 64, 8, 8, 64, [(1, 1, 1)]),
    "32 rows, split": ([(1, 1800)], 2, 2, 128, [(1, 1, 2)]),
    "32 rows, split, d 64": ([(1, 1800)], 2, 2, 64, [(1, 1, 2)]),
    "32 rows, many parts": ([(1, 5000)], 1, 1, 128, [(1, 1, 3)]),
    "32 rows, many parts, d 64": ([(1, 5000)], 1, 1, 64, [(1, 1, 3)]),
    "tiles of 32": ([(40, 200)] * 3, 4, 2, 128, [(1, 0, 1)]),
    "tiles of 32, d 64": ([(40, 200)] * 3, 4, 2, 64, [(1, 0, 1)]),
    "tiles of 32, many parts": ([(33, 6000)], 1, 1, 128, [(1, 0, 3)]),
    "tiles of 32, many parts, d 64": ([(33, 6000)], 1, 1, 64, [(1, 0, 3)]),
    "64 rows": ([(64, 1000)] * 32, 8, 8, 128, [(2, 1, 1)]),
    "64 rows, d 64": ([(64, 1000)] * 32, 8, 8, 64, [(2, 1, 1)]),
    "tiles of 64": ([(512, 2048)], 28, 4, 128, [(2, 0, 1)]),
    "tiles of 64, d 64": ([(100, 100)] * 64, 4, 4, 64, [(2, 0, 1)]),
    "tiles of 64, split": ([(700, 9000)], 2, 1, 128, [(2, 0, 2)]),
    "tiles of 64, split, d 64": ([(900, 12000)], 4, 1, 64, [(2, 0, 2)]),
    "128 rows": ([(100, 100)] * 64, 4, 4, 128, [(4, 1, 1)]),
    "tiles of 128": ([(300, 300)] * 16, 28, 4, 128, [(4, 0, 1)]),
    "tiles of 128, d 64": ([(300, 300)] * 16, 28, 4, 64, [(4, 0, 1)]),
    "tiles of 128, split": ([(700, 8300)], 8, 2, 128, [(4, 0, 2)]),
    "tiles of 128, split, d 64": ([(1500, 9000)], 8, 2, 64, [(4, 0, 2)]),
    "two launches": ([(1600, 2500)] + [(1, 60 * s + 1) for s in range(38)] + [(2, 2)], 16, 4, 128,
                     [(4, 0, 2), (1, 1, 1)]),
    "two launches, d 64": ([(1, 55 * s + 1) for s in range(69)] + [(4000, 4000)], 12, 4, 64,
                           [(4, 0, 2), (1, 1, 1)]),
}


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("amdclang++")
    if not cxx:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(HARNESS)
    subprocess.run([cxx, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2512_16229_amd", "csrc"),
                    str(d / "plan.cpp"), "-o", str(d / "plan")], check=True)

    def run(calls):
        """of each call fits, bytes and the launches (wm, single, slots, splits, chunk)"""
        text = "\n".join(" ".join(map(str, c)) for c in calls) + "\n"
        out = subprocess.run([str(d / "plan")], input=text, capture_output=True, text=True, check=True).stdout
        rows = [list(map(int, line.split())) for line in out.splitlines()]
        return [(r[0], r[1], [tuple(r[i:i + 5]) for i in range(2, len(r), 5)]) for r in rows]
    return run


def sizes(form):
    lens, heads, kv_heads, d, _ = FORMS[form]
    return heads, kv_heads, d, len(lens), sum(n for n, _ in lens), max(n for n, _ in lens), max(m for _, m in lens)


@pytest.mark.parametrize("form", FORMS)
def test_forms(plans, form):
    (fits, _, parts), = plans([sizes(form)])
    got = [(wm, single, 1 if splits == 1 else 2 if splits <= 16 else 3) for wm, single, _, splits, _ in parts]
    assert fits and got == FORMS[form][4], parts


def test_forms_reach_every_kernel():
    """Row tiles of 32, 64 and 128, written whole and joined, and both joining forms, at either head_dim."""
    seen = {(d, wm, splits > 1) for _, _, _, d, parts in FORMS.values() for wm, _, splits in parts}
    assert seen == {(d, wm, s) for d in (64, 128) for wm in (1, 2, 4) for s in (False, True)}
    joins = {(d, splits) for _, _, _, d, parts in FORMS.values() for _, _, splits in parts if splits > 1}
    assert joins == {(64, 2), (64, 3), (128, 2), (128, 3)}


def test_places_and_workspace(plans):
    """Over the range of sizes: the launches' row tiles have a place each, their chunks cover max_len,
    and the workspace holds all parts."""
    calls = []
    for heads, kv_heads in ((1, 1), (28, 4), (32, 32), (16, 1)):
        for d in (64, 128):
            for n_seq in (1, 3, 64, 700):
                for rows in (1, n_seq, 33 * n_seq, 33 * n_seq + 2, 5000):
                    for max_rows in (1, 31, 200, rows):
                        for max_len in (0, 1, 700, 40000):
                            calls.append((heads, kv_heads, d, n_seq, rows, max_rows, max_len))
    for c, (fits, size, parts) in zip(calls, plans(calls)):
        heads, kv_heads, d, n_seq, rows, max_rows, max_len = c
        G, most = heads // kv_heads, min(max_rows, rows) * (heads // kv_heads)
        assert fits and 1 <= len(parts) <= 2
        need = 0
        for wm, single, slots, splits, chunk in parts:
            bm = 32 * wm
            if len(parts) == 2 and (wm, single) == (1, 1):
                assert slots == n_seq  # of sequences of up to 32 (row, head) pairs
            else:
                assert slots == (n_seq if single else rows * G // bm + n_seq) and single == (most <= bm)
            assert splits * chunk >= max_len and (splits - 1) * chunk < max(1, max_len)
            need += slots * kv_heads * splits * bm * (d + 2) * 4 if splits > 1 else 0
        assert size == need, c
