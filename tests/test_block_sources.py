"""What a block's kernels may not leave to the compiler's choice, by reading the sources: the order in
which C++ evaluates the two sides of a product is open, so nothing that one side calls may write what
the other reads."""
import os
import re

from paper_2205_11048_gb300 import build as BLD
from tests.test_chained_loads import code_of, kernels


def lambdas(body):
    """(name, parameters, body) of every lambda that has a name."""
    for m in re.finditer(r"\bauto (\w+) = \[&\]\(([^)]*)\)\s*(?:->\s*\w+\s*)?\{", body):
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(body[i], 0)
            i += 1
        yield m.group(1), m.group(2), body[m.end():i - 1]


def test_parameters_are_read_into_the_lambdas_own_variables():
    found = 0
    for kernel, _, body in kernels(code_of(os.path.join(BLD.CSRC, "gba_resnorm.cu"))):
        for name, _, inner in lambdas(body):
            for into in re.findall(r"\bparams<1>\([^;]*?(\w+)\);", inner):
                found += 1
                assert re.search(r"\bfloat\b[^;]*\b%s\[1\]" % into, inner), (kernel, name, into)
    assert found >= 3
