"""Host-side checks of the assembly of the grouped linear layers (no GPU needed; skipped when
hipcc is absent).  Their loads to LDS and, on large tiles, their products are written out, and the
compiler does not know the wait states around an instruction that it did not choose.

 - A vector memory instruction may read a scalar register five wait states after a vector
   instruction wrote it, not before.
 - A product's sums may be read by anything but the next product of the same sums 18 wait states
   after it.  The loops end in 24; here: no instruction of a loop of products moves its sums.
 - The kernels keep their accumulators and fragments in registers: no scratch."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2505_17826_amd import build_lib as B

HIPCC = B.HIPCC if os.path.exists(B.HIPCC) else shutil.which("hipcc")
pytestmark = pytest.mark.skipif(not HIPCC, reason="hipcc not available")


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    texts = {}
    for src in ("k_linear.hip", "k_linear_few.hip"):
        out = tmp_path_factory.mktemp("s") / (src + ".s")
        cmd = [HIPCC, *[f for f in B.CFLAGS if f != "-fPIC"], *B.SOURCE_FLAGS.get(src, []),
               "--cuda-device-only", "-S", os.path.join(B.CSRC, src), "-o", str(out)]
        r = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
        assert r.returncode == 0, r.stderr[-2000:]
        texts[src] = out.read_text()
    return texts


def _regs(tok, kind):
    m = re.match(kind + r"\[(\d+):(\d+)\]$", tok)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1))
    m = re.match(kind + r"(\d+)$", tok)
    return {int(m.group(1))} if m else set()


def _lines(text):
    for line in text.splitlines():
        s = line.split(";")[0].strip()
        if s and not s.startswith("."):
            yield s


def early_reads(text):
    """Loads to LDS that read a scalar register less than five wait states after a vector
    instruction wrote it."""
    bad, before = [], []  # before: (wait states, scalar registers that a vector instruction wrote)
    for s in _lines(text):
        ops = [o for o in re.split(r"[\s,]+", s) if o]
        if s.endswith(":"):
            continue  # what falls through a label counts
        if ops[0].startswith("buffer_load") and "lds" in ops:
            used, states = _regs(ops[2], "s"), 0
            for n, regs in reversed(before):
                if regs & used and states < 5:
                    bad.append((before[-6:], s))
                states += n
                if states >= 5:
                    break
        n = int(ops[1], 0) + 1 if ops[0] == "s_nop" else 1
        wrote = set()
        if ops[0].startswith("v_") and len(ops) > 1:
            for o in ops[1:3] if ops[0].startswith(("v_cmp", "v_div_scale", "v_add_co", "v_sub_co")) else ops[1:2]:
                wrote |= _regs(o, "s")
        before = (before + [(n, wrote)])[-12:]
    return bad


def test_checker_flags_the_pattern():
    bad = "v_readlane_b32 s5, v1, 3\ns_mov_b32 m0, s9\ns_nop 0\nbuffer_load_dwordx4 v3, s[4:7], 0 offen lds\n"
    good = bad.replace("s_nop 0", "s_nop 4")
    assert len(early_reads(bad)) == 1 and not early_reads(good)
    assert not early_reads(bad.replace("s5,", "s12,"))


@pytest.mark.parametrize("src", ("k_linear.hip", "k_linear_few.hip"))
def test_loads_to_lds_wait_for_their_registers(asm, src):
    assert "lds" in asm[src]
    bad = early_reads(asm[src])
    assert not bad, bad[:2]


def test_sums_stay_in_place(asm):
    text = asm["k_linear.hip"]
    large = [n for n in re.findall(r"^(_ZN\w*5k_lin\w*):", text, re.M) if re.search(r"Li8ELi8E", n)]
    assert large
    for name in large:
        body = text[text.index("\n" + name + ":"):]
        body = body[:body.index(".Lfunc_end")]
        blocks = re.split(r"^\.LBB\w+:", body, flags=re.M)
        loops = [b for b in blocks if len(re.findall(r"v_mfma", b)) > 8]
        assert loops, name
        for b in loops:
            assert "accvgpr" not in b and not re.search(r"v_mov\S* .*\ba\[?\d", b), name
        assert re.search(r"s_nop 15\n\s*s_nop 7", body), name


@pytest.mark.parametrize("src", ("k_linear.hip", "k_linear_few.hip"))
def test_no_scratch(asm, src):
    kernels = re.findall(r"\.name:\s+(\S+).*?\.private_segment_fixed_size:\s+(\d+)", asm[src], re.S)
    assert kernels and not [k for k in kernels if int(k[1])]
