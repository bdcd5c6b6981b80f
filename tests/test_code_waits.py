"""Wait states in the built library's gfx950 code, which is disassembled.

The hardware does not wait by itself in some places, and the compiler does for instructions of its
own but not for those in assembly strings:
  a copy to LDS reads M0, which must have been written at least one wait state before;
  a memory instruction reads its address from scalar registers that a vector instruction must not
  have written in the five wait states before (every copy to LDS is looked at, along all ways that
  lead to it);
  a matrix instruction reads registers that a vector instruction must not have written in the two
  before, and of a 16x16x32 one the summand's registers must not be written in the three after."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2305_16317_amd as pd

OBJDUMP = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"
LINE = re.compile(r"^\t(\S+)\s*(.*?)\s*// ([0-9A-F]+):(.*)$")


def _scalars(text):
    out = set()
    for lo, hi, one in re.findall(r"\bs(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        out |= {int(one)} if one else set(range(int(lo), int(hi) + 1))
    return out


def _vectors(text):
    out = set()
    for lo, hi, one in re.findall(r"\bv(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        out |= {int(one)} if one else set(range(int(lo), int(hi) + 1))
    return out


def _scalars_written(name, ops):
    """Scalar registers that a vector instruction writes."""
    parts = ops.split(",")
    if name.startswith(("v_readfirstlane", "v_readlane", "v_cmp")):
        return _scalars(parts[0])
    if re.match(r"v_(mad_[ui]64|(add|sub|subrev)_co|(add|sub|subb|subbrev|addc)c?_co|div_scale)", name) and len(parts) > 1:
        return _scalars(parts[1])
    return set()


def _functions(listing):
    code = []
    for line in listing.splitlines():
        if line.endswith(">:"):
            if code:
                yield code
            code = []
            continue
        m = LINE.match(line)
        if m:
            to = re.search(r"<[^>]*?(?:\+0x([0-9a-f]+))?>$", m.group(4).strip())
            code.append((int(m.group(3), 16), m.group(1), m.group(2), None if to is None else int(to.group(1) or "0", 16)))
    if code:
        yield code


def _faults(code):
    """(copies to LDS, those with a wait missing) of a function [(address, name, operands, branch target)]."""
    is_copy = [("_lds_" in name and name.startswith("global_load")) or (name.startswith("buffer_load") and ops.endswith(" lds"))
               for _, name, ops, _ in code]
    if not any(is_copy):
        return 0, []
    at = {address: i for i, (address, *_) in enumerate(code)}
    jumps = {}
    for i, (_, name, _, to) in enumerate(code):
        if name.startswith(("s_branch", "s_cbranch")) and to is not None:
            jumps.setdefault(at[code[0][0] + to], []).append(i)

    def before(i):
        falls = i > 0 and code[i - 1][1] not in ("s_branch", "s_endpgm", "s_setpc_b64")
        return jumps.get(i, []) + ([i - 1] if falls else [])

    bad = []
    for i in (i for i, yes in enumerate(is_copy) if yes):
        reads = _scalars(code[i][2])
        ways, seen = [(j, 0) for j in before(i)], set()
        while ways:
            j, waited = way = ways.pop()
            if waited >= 5 or way in seen:
                continue
            seen.add(way)
            _, name, ops, _ = code[j]
            if (waited < 1 and name.startswith("s_") and ops.startswith("m0")) or reads & _scalars_written(name, ops):
                bad.append((hex(code[i][0]), name, ops, code[i][1], code[i][2]))
            step = waited + (int(ops, 0) + 1 if name == "s_nop" else 1)
            ways += [(k, step) for k in before(j)]
    return sum(is_copy), bad


def _matrix_faults(code):
    """(matrix instructions, pairs of a vector and a matrix instruction too close to each other)."""
    bad, count = [], 0
    split = [re.split(r",\s*(?![^\[]*\])", ops) for _, _, ops, _ in code]
    for i, (address, name, ops, _) in enumerate(code):
        if not name.startswith("v_mfma"):
            continue
        count += 1
        for way, most, regs in ((-1, 2, _vectors(",".join(split[i][1:]))),
                                (1, 3 if "16x16x32" in name else 0, _vectors(split[i][3]))):
            waited, j = 0, i + way
            while waited < most and 0 <= j < len(code) and not code[j][1].startswith(("s_branch", "s_cbranch")):
                other = code[j][1]
                if other.startswith("v_") and not other.startswith(("v_mfma", "v_accvgpr", "v_cmp")) and _vectors(split[j][0]) & regs:
                    bad.append((hex(address), name, ops, other, code[j][2]))
                waited += int(code[j][2], 0) + 1 if other == "s_nop" else 1
                j += way
    return count, bad


def _parse(text):
    return list(_functions("0 <f>:\n" + "\n".join(f"\t{ops} // {4 * i:08X}: 0" for i, ops in enumerate(text))))[0]


def test_the_check_sees_a_missing_wait():
    copy = "global_load_lds_dwordx4 v1, s[4:5]"
    assert _faults(_parse(["s_mov_b32 m0, s2", copy]))[1]
    assert not _faults(_parse(["s_mov_b32 m0, s2", "s_nop 0", copy]))[1]
    assert _faults(_parse(["v_readfirstlane_b32 s5, v3", "s_mov_b32 m0, s2", "s_nop 2", copy]))[1]
    assert not _faults(_parse(["v_readfirstlane_b32 s5, v3", "s_mov_b32 m0, s2", "s_nop 3", copy]))[1]
    assert not _faults(_parse(["v_readfirstlane_b32 s6, v3", "s_mov_b32 m0, s2", "s_nop 0", copy]))[1]


def test_the_check_sees_a_vector_instruction_too_close_to_a_matrix_one():
    mfma, cvt = "v_mfma_f32_16x16x32_f16 v[8:11], v[4:7], v[0:3], v[12:15]", "v_cvt_pk_f16_f32 v%d, v20, v21"
    assert _matrix_faults(_parse([cvt % 3, "s_nop 0", mfma]))[1]
    assert not _matrix_faults(_parse([cvt % 3, "s_nop 1", mfma]))[1]
    assert _matrix_faults(_parse([mfma, "s_nop 1", cvt % 12]))[1]
    assert not _matrix_faults(_parse([mfma, "s_nop 2", cvt % 12]))[1]


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    tmp_path = tmp_path_factory.mktemp("code")
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    pd.load()
    lib = shutil.copy(os.path.join(os.path.dirname(pd.__file__), "libparadigms.so"), tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", str(lib)], check=True, capture_output=True, cwd=tmp_path)
    parts = sorted(p for p in tmp_path.iterdir() if p.name.endswith("gfx950"))
    assert parts
    return [subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(p)], check=True, capture_output=True, text=True).stdout
            for p in parts]


def test_copies_to_lds_wait_for_what_they_read(listings):
    copies = 0
    for listing in listings:
        for code in _functions(listing):
            count, bad = _faults(code)
            copies += count
            assert not bad, bad[:3]
    assert copies > 1000          # the attention kernels and the convolutions are among them


def test_vector_instructions_keep_their_distance_to_matrix_ones(listings):
    products = 0
    for listing in listings:
        for code in _functions(listing):
            count, bad = _matrix_faults(code)
            products += count
            assert not bad, bad[:3]
    assert products > 1000
