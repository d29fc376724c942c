"""What the inline assembly of the operators' kernels rests on and does not tell the compiler, read from the assembly that it makes of them."""
import importlib.util
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lines(tmp_path_factory):
    """Labels and instructions of zf_head.hip's kernels."""
    spec = importlib.util.spec_from_file_location("zapformat_build", os.path.join(ROOT, "paper_2506_01151_amd", "build.py"))
    builder = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(builder)
    out = str(tmp_path_factory.mktemp("asm") / "head.s")
    rc, err = builder._run(["hipcc", "-x", "hip", "--offload-device-only", "-S", os.path.join(builder.CSRC, "zf_head.hip"), "-o", out] + [f for f in builder.FLAGS if f != "-fPIC"])
    assert rc == 0, err
    text = [l.split(";")[0].strip() for l in open(out)]
    return [l for l in text if l and not l.startswith("//") and (not l.startswith(".") or l.startswith(".LBB"))]


def test_nothing_but_the_loads_into_lds_uses_m0(lines):
    """Loads straight into LDS take their place from m0, which inline assembly writes for each of them: it cannot be named as overwritten there (m0 is reserved), so the compiler's own
    instructions may not use it in these kernels."""
    loads = [k for k, l in enumerate(lines) if l.startswith("global_load_lds")]
    own = {k - 2 for k in loads}
    assert loads and all(re.fullmatch(r"s_mov_b32 m0, s\d+", lines[k - 2]) and lines[k - 1] == "s_nop 0" for k in loads)
    other = [l for k, l in enumerate(lines) if re.search(r"\bm0\b|movrel|sendmsg|_gws_", l) and k not in own]
    assert not other, other[:5]


def scalars(text):
    out = {int(n) for n in re.findall(r"\bs(\d+)\b", text)}
    for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", text):
        out |= set(range(int(a), int(b) + 1))
    return out


def test_addresses_of_loads_into_lds_have_settled(lines):
    """A vector instruction's scalar result may be a load's address five wait states later, which the compiler sees to for instructions that it knows, not for those of inline assembly."""
    jumps = {}
    for k, l in enumerate(lines):
        m = re.match(r"s_c?branch\S*\s+(\.LBB\w+)", l)
        if m:
            jumps.setdefault(m[1], []).append(k)

    def written(k, states, address, seen):                 # on every way to place k, fewer than five states back
        while k >= 0 and states < 5:
            l = lines[k]
            if l.startswith(".LBB"):
                for j in jumps.get(l.rstrip(":"), []):
                    if (j, states) not in seen:
                        seen.add((j, states))
                        yield from written(j, states, address, seen)
                if lines[k - 1].startswith(("s_branch", "s_endpgm")):
                    return
            else:
                op = l.split()
                if op[0].startswith("v_") and scalars(op[1]) & address:
                    yield l
                states += int(op[1]) + 1 if op[0] == "s_nop" else 1
            k -= 1

    loads = [k for k, l in enumerate(lines) if l.startswith("global_load_lds")]
    bad = [(lines[k], l) for k in loads for l in written(k - 1, 0, scalars(lines[k]), set())]
    assert any(scalars(lines[k]) for k in loads) and not bad, bad[:5]
