"""Guards on the generated code of the paged cache's kernels (no GPU needed): nothing is spilled, and as many waves a SIMD as the cuts reckon with."""
import re

import pytest

from test_isa_guards import _assembly, _instructions


def _kernels(text, name):
    for s in (i for i, l in enumerate(text) if re.match(r"^_ZN2bc\w*%s\w+:" % name, l)):
        e = next(i for i in range(s, len(text)) if text[i].startswith(".Lfunc_end"))
        waves = next(int(x.group(1)) for x in (re.match(r"; Occupancy: (\d+)", l) for l in text[e:]) if x)
        yield text[s].split(":")[0], _instructions(text[s:e]), waves


@pytest.fixture(scope="module")
def attend(tmp_path_factory):
    return _assembly("bc_paged_attend.hip", tmp_path_factory.mktemp("attend"))


def test_attend_spills_nothing(attend):
    few, many = list(_kernels(attend, "paged_few_kernel")), list(_kernels(attend, "paged_many_kernel"))
    assert len(few) == 16 and len(many) == 4
    for name, body, waves in few + many:
        assert not any(l.startswith("scratch_") for l in body), name
        # (one tile of columns and four waves a workgroup: four workgroups a compute unit; the others two waves a SIMD)
        assert waves >= (4 if "Li1ELi4E" in name else 2), (name, waves)


def test_append_spills_nothing(tmp_path):
    text = _assembly("bc_paged_append.hip", tmp_path)
    found = list(_kernels(text, "paged_append_kernel")) + list(_kernels(text, "paged_append_one_kernel"))
    assert len(found) == 16 + 8
    for name, body, _ in found:
        assert not any(l.startswith("scratch_") for l in body), name
