"""What the serving kernels do when a bounded wait runs out, and with what they read then: read from the sources or run on the host, as
making one run out would leave a GPU with work of a block that has ended."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_26558_b200", "csrc")


def _code(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_a_block_that_gives_up_waits_for_the_answer_it_asked_for():
    """The hardware's answer to clusterlaunchcontrol is 16 bytes written to the block's shared memory: every way out waits for it."""
    code = _code("shared_stream.cuh")
    loop = code.index("for (; cta >= 0 && ok;") if "for (; cta >= 0 && ok;" in code else code.index("for (int cta = blockIdx.x")
    after = code[loop:code.index("if (a.behind_tc) pdl_wait();", loop)]
    failed = after[after.rindex("if (!ok)"):]
    assert re.search(r"mbar_wait_bounded\(&answered, ", failed), failed


def test_a_meeting_that_runs_out_is_not_passed_over():
    """Warps that edit a tile together may not go on as if the others had come: the wait flags the status, as every other one does."""
    code = _code("shared_stream.cuh")
    body = code[code.index("auto meeting ="):]
    assert re.search(r"if \(!mbar_wait_bounded\(&meet\[set\], phase\)\) met = false;", body[:body.index("\n                };")]), body[:400]
    last = body[body.index("meeting(1);"):]
    assert re.search(r"!__all_sync\(0xffffffffu, met\)\) \{\s*ok = false;[^}]*CASS_ERR_TIMEOUT", last[:500]), last[:500]


def test_tensor_memory_is_freed_behind_the_products():
    """Whether its waits ran out or not, the thread that issued products waits for the last of them before its block frees tensor memory."""
    code = _code("shared_attn_tc.cu")
    issue = code[code.index("if (tc_elect()) {"):code.index("} else {\n        asm volatile(\"setmaxnreg.inc")]
    end = issue[issue.rindex("tc_commit("):]
    assert re.search(r"tc_commit\((\w+)\);\s*mbar_wait_bounded\(\1, 0\);", end), end
    assert "if (ok)" not in end.split("mbar_wait_bounded")[0], end


# Ranges of parts as the table may hold them: written, never written (whatever the scratch held), half written.
_SLOTS = r"""
#include <cstdio>
#include <random>
#include "shared_attn.cuh"
int main() {
    std::mt19937 rng(1);
    long kept = 0, bad = 0, cut = 0;
    for (int n : {1, 2, 450, 1 << 20})
        for (int i = 0; i < 100000; ++i) {
            int2 s = make_int2((int)rng(), (int)rng());
            if (i % 3 == 0) s = make_int2((int)(rng() % n), (int)(rng() % n));
            if (i % 1000 == 1) s = make_int2(0, n - 1);
            if (i % 1000 == 2) s = make_int2(0, n);
            if (i % 1000 == 4) s = make_int2(-1, 0);
            const int2 t = cass::shared_slots(s, n);
            const bool fine = s.x >= 0 && s.y < n && s.x <= s.y;
            if (fine ? t.x != s.x || t.y != s.y : t.y - t.x + 1 != 0 || t.x < 0) ++bad;
            ++(fine ? kept : cut);
        }
    std::printf("%ld %d %d\n", bad, kept > 1000, cut > 1000);
}
"""


def test_parts_that_were_never_written_are_not_read(tmp_path):
    """The merge reads where a segment's parts lie from the scratch.  If the kernel before it gave up, that is whatever was there: a range
    outside the parts counts as none."""
    import test_first_calls
    assert test_first_calls._output(tmp_path, _SLOTS) == ["0", "1", "1"]
    code = _code("shared_attn.cu")
    reads = re.findall(r"[^;]*\ba\.slots\[[^;]*;", code)
    assert reads and all("shared_slots(" in r for r in reads), reads
