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
    body = code[code.index("auto sync_set ="):]
    body = body[:body.index("\n                };")]
    assert "mbar_wait_bounded" not in body and re.search(r"\bwait\(&meet\[set\], ", body), body


def test_tensor_memory_is_freed_behind_the_products():
    """Whether its waits ran out or not, the thread that issued products waits for the last of them before its block frees tensor memory."""
    code = _code("shared_attn_tc.cu")
    issue = code[code.index("if (tc_elect()) {"):code.index("} else {\n        asm volatile(\"setmaxnreg.inc")]
    end = issue[issue.rindex("tc_commit("):]
    assert re.search(r"tc_commit\((\w+)\);\s*mbar_wait_bounded\(\1, 0\);", end), end
    assert "if (ok)" not in end.split("mbar_wait_bounded")[0], end
