"""fef_draw_logits writes some places of a row twice: -inf first, then what turns out to be kept, by other wavefronts.  Whatever way a kernel takes, the
first stores have landed (their wavefront has waited for all of its own, and the workgroup has met at a barrier behind that) before the second ones
are made.  Looked up in the assembly of this repository's own sources; no GPU."""
import os
import re

import pytest

from paper_2605_14305_amd import build as b

AGAIN = "written again"  # the comment in the assembly in front of stores to places that are written already


def _kernels(lines):
    """{name: (instructions, labels)}; an instruction is its text, comments that hold AGAIN among them."""
    found = {}
    for start in (i for i, l in enumerate(lines) if re.match(r"^_Z\w*draw_\w*kernel\w*:", l)):
        code, labels = [], {}
        for line in lines[start + 1:]:
            if line.startswith(".Lfunc_end"):
                break
            t = line.split(";")[0].strip()
            if re.match(r"^\.?[A-Za-z_][\w.$]*:", t):
                labels[t.split(":")[0]] = len(code)
            elif t and not t.startswith((".", "#")):
                code.append(t)
            elif AGAIN in line:
                code.append(AGAIN)
        found[lines[start].split(":")[0]] = code, labels
    return found


def unwaited(code, labels):
    """Stores from which a way leads to AGAIN without a wait for stores and a barrier behind it."""
    bad = []
    for at in (i for i, t in enumerate(code) if t.startswith(("global_store", "flat_store"))):
        seen, ways = set(), [(at + 1, False)]
        while ways:
            i, landed = ways.pop()
            if i >= len(code) or (i, landed) in seen:
                continue
            seen.add((i, landed))
            t = code[i]
            if t == AGAIN:
                bad.append(at)
                break
            if t.startswith("s_barrier") and landed:
                continue
            if t.startswith("s_waitcnt") and "vmcnt(0)" in t:
                landed = True
            elif t.startswith(("global_store", "flat_store")):
                continue  # looked at for itself
            if t.startswith("s_endpgm"):
                continue
            if t.startswith(("s_branch", "s_cbranch")):
                ways.append((labels[t.split()[1]], landed))
            if not t.startswith("s_branch"):
                ways.append((i + 1, landed))
    return bad


@pytest.mark.parametrize("body,bad", [
    (["global_store_dword v0, v1, s[0:1]", "s_barrier", AGAIN], [0]),
    (["global_store_dword v0, v1, s[0:1]", "s_waitcnt lgkmcnt(0)", "s_barrier", AGAIN], [0]),
    (["global_store_dword v0, v1, s[0:1]", "s_waitcnt vmcnt(0)", AGAIN], [0]),
    (["global_store_dword v0, v1, s[0:1]", "s_waitcnt vmcnt(0) lgkmcnt(0)", "s_barrier", AGAIN], []),
    (["global_store_dword v0, v1, s[0:1]", "s_cbranch_vccz .LBB0_1", "s_waitcnt vmcnt(0)", "s_barrier", AGAIN], [0]),
    (["global_store_dword v0, v1, s[0:1]", "s_waitcnt vmcnt(0)", "s_barrier", "global_store_dword v0, v1, s[0:1]", AGAIN], [3]),
])
def test_what_is_looked_for(body, bad):
    assert unwaited(body, {".LBB0_1": len(body) - 1}) == bad


@pytest.mark.skipif(not os.path.exists(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")), reason="no compiler")
def test_stores_have_landed_before_places_are_written_again():
    kernels = _kernels(b._assembly("draw_kernels.hip"))
    twice = {name for name, (code, _) in kernels.items() if AGAIN in code}
    for part, count in (("draw_rows_kernel", 4), ("draw_left_kernel", 2), ("draw_finish_kernel", 2)):
        assert sum(part in name for name in twice) == count, part
    for name in twice:
        code, labels = kernels[name]
        assert not unwaited(code, labels), (name, [code[i] for i in unwaited(code, labels)][:4])
