"""Host checks on the sources of the operators around the split layer."""
import ast
import os
import re

from paper_2011_09208_amd import buildlib


def _arguments(text):
    """The arguments of every raw buffer load or store in `text`."""
    for m in re.finditer(r"__builtin_amdgcn_raw_buffer_(?:load|store)_\w+\(", text):
        depth, args, last = 1, [], m.end()
        for i in range(m.end(), len(text)):
            depth += (text[i] in "([{") - (text[i] in ")]}")
            if depth == 0 or (depth == 1 and text[i] == ","):
                args.append(text[last:i].strip())
                last = i + 1
            if depth == 0:
                break
        yield args


def test_no_buffer_load_is_put_out_of_range_by_its_scalar_offset():
    """Compilers describe the scalar offset of a raw buffer load as outside of the range check.  It may carry a step's first byte; what is
    to read nothing is marked in the lanes' offsets or has no records."""
    text = open(os.path.join(buildlib.PKG, "csrc", "w4.hip")).read()
    found = list(_arguments(text))
    assert len(found) >= 5
    for rsrc, lane, scalar, flags in found:
        assert scalar in ("0", "k >> 1", "k >> 5"), (rsrc, lane, scalar)
    limit = re.search(r"#define\s+WS_W4_MAX_CLASSES\s+\(\(1 << 30\) - (\d+)\)", open(buildlib.DEPS[-1]).read())
    assert 4 * ((1 << 30) - int(limit.group(1))) <= (1 << 32) - 1024               # the mark is beyond the largest shard's biases


def test_the_benchmark_reads_what_it_counts():
    """The norm's call is counted with the bytes of a stream and of an addition to it: two buffers, not one read twice."""
    tree = ast.parse(open(os.path.join(os.path.dirname(buildlib.PKG), "bench.py")).read())
    calls = [n for n in ast.walk(tree) if isinstance(n, ast.Call) and getattr(n.func, "attr", "") == "rms_norm_fwd"]
    assert calls
    for call in calls:
        buffers = [a.id for a in call.args if isinstance(a, ast.Name)]
        assert len(set(buffers)) == len(buffers), buffers
