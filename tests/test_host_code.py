"""Properties of the built device code, from the metadata that the compiler leaves in libkperf.so, and of the binding, both without a GPU."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
READELF = "/opt/rocm/llvm/bin/llvm-readelf"


def kernels(tmp_path):
    """{mangled name: bytes of scratch memory per lane} of every kernel in the library."""
    lib = os.path.join(ROOT, "paper_2505_21661_amd", "libkperf.so")
    if not os.path.exists(lib):
        from paper_2505_21661_amd import build as kbuild

        kbuild.build()
    data = open(lib, "rb").read()
    found = {}
    at = data.find(b"\x7fELF", 1)
    while at >= 0:
        end = data.find(b"\x7fELF", at + 1)
        path = tmp_path / "code.o"
        path.write_bytes(data[at:end if end >= 0 else len(data)])
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True).stdout
        for entry in notes.split("- .agpr_count:")[1:]:
            found[re.search(r"\.name: +(\S+)", entry).group(1)] = int(re.search(r"\.private_segment_fixed_size: +(\d+)", entry).group(1))
        at = end
    return found


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_replay_kernels_hold_their_state_in_registers(tmp_path):
    """The bounds on hardware waves per SIMD leave every replay kernel the vector registers that it needs."""
    found = {k: v for k, v in kernels(tmp_path).items() if "kp_waits_main" in k or "kp_pairs_main" in k}
    assert len(found) == 14, found  # five forms of the wait kernel, nine of the timeline kernel
    assert not any(found.values()), found


@pytest.mark.parametrize("raw_lookup", [True, False])
def test_a_call_without_a_stream_takes_torchs_current_one(monkeypatch, raw_lookup):
    """With torch's lookup of the bare handle, and by its public interface where a torch does not have that."""
    torch = pytest.importorskip("torch")
    from paper_2505_21661_amd import binding

    class Stream:
        cuda_stream = 0x5000

    monkeypatch.setattr(torch.cuda, "init", lambda: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Stream)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x4000 + device, raising=False)
    if not raw_lookup:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    monkeypatch.setattr(binding, "_current_stream", None, raising=False)
    assert binding._stream(None) == (0x4003 if raw_lookup else 0x5000)
    assert binding._stream(None) == (0x4003 if raw_lookup else 0x5000)
    assert binding._stream(7) == 7 and binding._stream(Stream) == 0x5000


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_every_kernel_of_the_statistics_is_taken_by_some_geometry(tmp_path):
    """Either side of the lines in the numbers of workgroups and regions, all waves and ring sizes."""
    from tests import fake_hip

    calls = [{"fn": "kp_trace_reduce_hdr", "trace": (n_wg, waves, regions, 1 << log2)} for n_wg in (1, 257, 401, 1401, 2600)
             for waves in range(1, 17) for regions in (1, 8, 9, 16, 17, 32, 33, 64, 65, 128) for log2 in range(1, 20)]
    taken = {x[0] for _, launches in fake_hip.run(calls, tmp_path) for x in launches}
    built = {k for k in kernels(tmp_path) if "kp_reduce" in k}
    assert built and built == taken, built ^ taken


OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def touched_in_flight(code):
    """Of a kernel's instructions (address, text, address that it may branch to): the number of clock samples, and what names a sample's
    scalar registers on some path before the wait that lets it land."""
    def registers(text):
        out = {int(a) for a in re.findall(r"(?<![\w\[:])s(\d+)\b", text)}
        for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", text):
            out |= set(range(int(a), int(b) + 1))
        return out

    number = {at: n for n, (at, _, _) in enumerate(code)}
    samples, touched = 0, []
    for n, (_, text, _) in enumerate(code):
        m = re.match(r"s_mem(?:real)?time s\[(\d+):(\d+)\]", text)
        if not m:
            continue
        samples += 1
        mine, todo, been = set(range(int(m[1]), int(m[2]) + 1)), [n + 1], set()
        while todo:
            at = todo.pop()
            while at < len(code) and at not in been:
                been.add(at)
                _, x, target = code[at]
                if x.startswith("s_endpgm") or (x.startswith("s_waitcnt") and "lgkmcnt(0)" in x):
                    break
                if registers(x) & mine:
                    touched.append((text, x))
                    break
                if x.startswith("s_cbranch"):
                    todo.append(number[target])
                if x.startswith("s_branch"):
                    at = number[target]
                else:
                    at += 1
    return samples, touched


def disassembly(tmp_path, name):
    """{mangled name: its instructions} of the library's kernels with `name` in theirs."""
    if not os.path.exists(os.path.join(ROOT, "paper_2505_21661_amd", "libkperf.so")):
        from paper_2505_21661_amd import build as kbuild

        kbuild.build()
    data = open(os.path.join(ROOT, "paper_2505_21661_amd", "libkperf.so"), "rb").read()
    found, at = {}, data.find(b"\x7fELF", 1)
    while at >= 0:
        end = data.find(b"\x7fELF", at + 1)
        part = data[at:end if end >= 0 else len(data)]
        at = end
        if name.encode() not in part:
            continue
        path = tmp_path / "code.o"
        path.write_bytes(part)
        text = subprocess.run([OBJDUMP, "-d", str(path)], capture_output=True, text=True).stdout
        for begin, kernel, body in re.findall(r"^([0-9a-f]+) <(\S+)>:\n((?:.+\n?)*)", text, re.M):
            if name not in kernel:
                continue
            lines = []
            for line in body.splitlines():
                m = re.match(r"\s+(\S.*?)\s*// ([0-9A-F]+): \S+(?: \S+)*?(?: <(\S+?)(?:\+0x([0-9a-f]+))?>)?$", line)
                if m:
                    lines.append((int(m[2], 16), m[1], int(begin, 16) + int(m[4] or "0", 16) if m[3] else None))
            found[kernel] = lines
    return found


def test_the_paths_of_a_sample_are_followed():
    """What the next test takes for touched: a copy ahead of the wait, also behind a branch; not one behind it, nor other registers."""
    body = [(0, "s_memtime s[4:5]", None), (8, "s_cbranch_scc1 2", 24), (12, "s_waitcnt lgkmcnt(0)", None), (16, "s_mov_b32 s9, s4", None), (20, "s_endpgm", None),
            (24, "s_mov_b32 s9, s3", None), (28, "s_branch 4", 12)]
    assert touched_in_flight(body) == (1, [])
    body[5] = (24, "v_writelane_b32 v3, s5, 2", None)
    assert touched_in_flight(body) == (1, [("s_memtime s[4:5]", "v_writelane_b32 v3, s5, 2")])
    body[5] = (24, "s_load_dwordx4 s[0:3], s[8:9], 0x0", None)
    assert touched_in_flight(body) == (1, [])
    body[5] = (24, "s_load_dwordx4 s[4:7], s[8:9], 0x0", None)
    assert len(touched_in_flight(body)[1]) == 1


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
@pytest.mark.parametrize("kernel,places", [("kp_attn_tile", 5), ("kp_attn_few", 3), ("kp_attn_drafts", 2)])
def test_recorded_attentions_leave_a_sample_alone_until_it_lands(tmp_path, kernel, places):
    """A record site asks for the clock and does not wait; the compiler takes the registers as written at once, and may move or spill them."""
    recorded = {k: v for k, v in disassembly(tmp_path, kernel).items() if re.search(r"ELi[13]EEE", k)}
    assert len(recorded) == 8 * places, sorted(recorded)  # two clocks, types and sizes, for each place that keys may be in
    for name, lines in recorded.items():
        samples, touched = touched_in_flight(lines)
        assert samples >= 6 and not touched, (name, touched)
