"""Where the kernels of the operators on a paged cache keep what does not fit their registers.  Nothing in scratch memory: the build refuses that.
Scalars, which are every lane's, go to single lanes of vector registers; such a register, copied or overwritten where some lanes are off, would
give back other scalars, addresses among them: in the code that is built none is touched by anything but the reads and writes of its lanes."""
import os
import re
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIBRARY = os.path.join(ROOT, "paper_2510_23264_amd", "libpahq.so")
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(data):
    """The gfx950 code objects in the library: every bundle is its magic, a count, and (offset, size, length of a name, name) of each."""
    at = data.find(MAGIC)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + 24)
        entry = at + 32
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            if b"gfx950" in data[entry + 24:entry + 24 + length] and size:
                yield data[at + offset:at + offset + size]
            entry += 24 + length
        at = data.find(MAGIC, at + 24)


def vector_registers(text):
    out = set()
    for lo, hi, one in re.findall(r"(?<![\w.])v(?:\[(\d+):(\d+)\]|(\d+))(?!\w)", text):
        out.update(range(int(lo), int(hi) + 1) if lo else [int(one)])
    return out


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Instructions of every kernel on a paged cache, from the library that runs."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no tool to read code objects")
    path, out = tmp_path_factory.mktemp("code") / "code", {}
    for code in code_objects(open(LIBRARY, "rb").read()):
        if b"kv_few_k" not in code and b"kv_keep_k" not in code:
            continue
        path.write_bytes(code)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], stdout=subprocess.PIPE, text=True, check=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]+ <)", text):
            name = re.match(r"[0-9a-f]+ <(_ZN4pahq\d+kv_\w+)>:", part)
            if name:
                out[name.group(1)] = [line.split("//")[0].strip() for line in part.split("\n")[1:] if line.strip()]
    return out


def test_every_kernel_is_looked_at(kernels):
    found = sorted(re.match(r"_ZN4pahq\d+(kv_[a-z]+_k)", k).group(1) for k in kernels)
    assert {k: found.count(k) for k in set(found)} == {"kv_few_k": 9 + 2 * 10, "kv_tile_k": 2 + 2 * 3, "kv_join_k": 3, "kv_append_k": 6, "kv_keep_k": 1}


def test_scalars_kept_in_lanes_stay_what_they_are(kernels):
    kept = 0
    for name, code in kernels.items():
        lanes = set()
        for line in code:
            if line.startswith("v_writelane_b32"):
                lanes |= vector_registers(line.split(",")[0])
        kept += len(lanes)
        for line in code:
            if not line.startswith(("v_writelane_b32", "v_readlane_b32")):
                assert not vector_registers(line) & lanes, (name, line)
    assert kept >= 30                                    # there are such registers


def test_nothing_is_kept_in_scratch_memory(kernels):
    for name, code in kernels.items():
        assert not [line for line in code if line.startswith(("scratch_", "buffer_"))], name


def test_nothing_but_requests_into_lds_uses_their_base(kernels):
    """M0 is set just in front of every request into LDS, and by nothing else."""
    asked = 0
    for name, code in kernels.items():
        for i, line in enumerate(code):
            if "lds_dword" in line:
                asked += 1
                assert any(x.startswith("s_mov_b32 m0") for x in code[i - 2:i]), (name, code[i - 3:i + 1])
            elif re.search(r"\bm0\b", line):
                assert line.startswith("s_mov_b32 m0") and any("lds_dword" in x for x in code[i + 1:i + 3]), (name, line)
    assert asked > 100


def test_the_build_refuses_scratch_memory(monkeypatch, tmp_path):
    from paper_2510_23264_amd import build as b
    remark = "k.hip:1:1: remark: Function Name: %s [-R]\nk.hip:1:1: remark:     ScratchSize [bytes/lane]: %d [-R]\nk.hip:1:1: remark:     Dynamic Stack: %s [-R]\n"
    assert b.scratch_of(remark % ("a", 0, "False") + remark % ("b", 0, "False")) == {}
    assert b.scratch_of(remark % ("a", 0, "False") + remark % ("b", 12, "False")) == {"b": 12}
    assert b.scratch_of(remark % ("a", 0, "True")) == {"a": 0}
    assert b.NO_SCRATCH <= set(b.SOURCES)
    monkeypatch.setattr(b, "HERE", str(tmp_path))
    (tmp_path / "_build").mkdir()
    said = {"text": ""}

    def run(command, **how):
        open(command[-1], "w").close()
        return subprocess.CompletedProcess(command, 0, stdout=said["text"].encode())
    monkeypatch.setattr(subprocess, "run", run)
    for text, fine in ((remark % ("a", 0, "False"), True), (remark % ("a", 8, "False"), False), ("", False)):
        said["text"] = text
        if fine:
            assert b._compile("kv_attention.hip") == str(tmp_path / "_build" / "kv_attention.o")
        else:
            with pytest.raises(RuntimeError, match="scratch"):
                b._compile("kv_attention.hip")
            assert not (tmp_path / "_build" / "kv_attention.o").exists()
    assert b._compile("rows.hip")                        # others may
