"""What the inline assembly of the operators' kernels rests on and does not tell the compiler, read from the assembly that it makes of them."""
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_nothing_but_the_loads_into_lds_uses_m0(tmp_path):
    """Loads straight into LDS take their place from m0, which inline assembly writes for each of them: it cannot be named as overwritten there (m0 is reserved), so the compiler's own
    instructions may not use it in these kernels."""
    import importlib.util
    spec = importlib.util.spec_from_file_location("zapformat_build", os.path.join(ROOT, "paper_2506_01151_amd", "build.py"))
    builder = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(builder)
    out = str(tmp_path / "head.s")
    rc, err = builder._run(["hipcc", "-x", "hip", "--offload-device-only", "-S", os.path.join(builder.CSRC, "zf_head.hip"), "-o", out] + [f for f in builder.FLAGS if f != "-fPIC"])
    assert rc == 0, err
    lines = [l.split(";")[0].strip() for l in open(out)]
    lines = [l for l in lines if l and not l.startswith((".", "//"))]
    loads = [k for k, l in enumerate(lines) if l.startswith("global_load_lds")]
    own = {k - 2 for k in loads}
    assert loads and all(re.fullmatch(r"s_mov_b32 m0, s\d+", lines[k - 2]) and lines[k - 1] == "s_nop 0" for k in loads)
    other = [l for k, l in enumerate(lines) if re.search(r"\bm0\b|movrel|sendmsg|_gws_", l) and k not in own and not l.startswith("s_sendmsg sendmsg(MSG_DEALLOC_VGPRS)")]
    assert not other, other[:5]
