"""Guards on the generated code of the prompt step's kernels, as on the prefill kernels' (no GPU needed)."""
import re

import pytest

from test_isa_guards import HAND, _arguments, _assembly, _instructions, check_m0


@pytest.fixture(scope="module")
def text(tmp_path_factory):
    return _assembly("bc_prompt.hip", tmp_path_factory.mktemp("prompt"))


@pytest.mark.parametrize("kernel,wide,narrow", [("prompt_attn_kernel", 3, 4), ("prompt_few_kernel", 1, 2)])
def test_loads_to_lds_and_registers(text, kernel, wide, narrow):
    starts = [i for i, l in enumerate(text) if re.match(r"^_ZN2bc\w*%s\w+:" % kernel, l)]
    assert len(starts) == 2
    for s in starts:
        e = next(i for i in range(s, len(text)) if text[i].startswith(".Lfunc_end"))
        marked = _instructions(text[s:e])
        body = [l[:-len(HAND)] if l.endswith(HAND) else l for l in marked]
        assert check_m0(body) >= 4, text[s][:80]
        assert all("load_lds" in l for l in marked if l.endswith(HAND) and l.startswith("global_load")), text[s][:80]
        assert not any(l.startswith(("scratch_", "buffer_")) for l in body), text[s][:80]
        waves = next(int(x.group(1)) for x in (re.match(r"; Occupancy: (\d+)", l) for l in text[e:]) if x)
        assert waves >= (wide if "ILi128E" in text[s] else narrow), (text[s][:80], waves)


def test_the_chunks_are_found_behind_the_start_of_the_arguments(text):
    kernels = {k: a for k, a in _arguments(text).items() if "Params" in k}
    assert len(kernels) == 12 and all(a == [(0, "by_value")] for a in kernels.values()), kernels
