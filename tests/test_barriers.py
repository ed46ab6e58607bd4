"""A meeting of a workgroup that is asked for by the bare instruction says nothing to the compiler about memory: it may move ordinary reads of LDS from behind the meeting to before
it, where what other wavefronts' loads bring is not there yet.  Each has a fence for the compiler right behind it, and before it a wait that is one (no GPU needed)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2009_13003_amd", "csrc")


def test_a_fence_on_either_side_of_every_bare_meeting():
    found = 0
    for name in sorted(os.listdir(CSRC)):
        code = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        for m in re.finditer(r"__builtin_amdgcn_s_barrier\(\);", code):
            found += 1
            line = "%s:%d" % (name, code[:m.start()].count("\n") + 1)
            assert re.match(r'\s*asm volatile\("" ::: "memory"\);', code[m.end():]), line + ": no fence behind it"
            before = code[:m.start()].split(";")[-2]
            assert "wait_loads<" in before or ("s_waitcnt" in before and '"memory"' in before), line + ": no wait before it"
    assert found >= 3
