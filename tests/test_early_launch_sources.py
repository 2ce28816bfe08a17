"""Kernels that are set up while the kernel before them runs (launch_early) read what that kernel writes.  A
__restrict__ parameter promises the compiler that nobody else writes it while the kernel lives, which is false for
them, and lets it move loads above the wait: so they have none.  Read from the sources; no GPU needed."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_11430_b200", "csrc")


def _code(path):
    """A source file without its comments."""
    with open(path) as f:
        return re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)


def _signatures(code):
    """Name -> text from the kernel's __global__ to the brace that opens its body."""
    return {m.group(1): m.group(0) for m in re.finditer(r"__global__[^{;]*?\b(\w+_kernel)\s*\([^{]*\{", code)}


def _early(code):
    """Names of the kernels that are launched early: named in the call, or by the variable that it takes."""
    names = set()
    for what in re.findall(r"\blaunch_early\(\s*(\w+)", code):
        if what.endswith("_kernel"):
            names.add(what)
        names.update(re.findall(r"\bauto\s+%s\s*=\s*(\w+_kernel)" % what, code))
    return names


def _all():
    return {path: _code(path) for path in sorted(glob.glob(os.path.join(CSRC, "*.cu")))}


def test_the_early_kernels_are_found():
    early = set().union(*(_early(code) for code in _all().values()))
    assert early == {"rotary_write_kernel", "tree_commit_kernel", "token_attention_kernel", "token_attention_join_kernel"}


def test_no_early_kernel_promises_that_nobody_else_writes_its_arguments():
    for path, code in _all().items():
        signatures = _signatures(code)
        for name in _early(code):
            assert "__restrict__" not in signatures[name], f"{name} in {os.path.basename(path)}"


def test_every_early_kernel_waits():
    for path, code in _all().items():
        for name in _early(code):
            at = code.index(_signatures(code)[name])
            end = code.find("__global__", at + 1)
            assert "wait_for_previous();" in code[at:end if end > 0 else len(code)], name
