"""Rotation, cache rows and paged attention through the bounds-checked debugging build: no index misses its extent, and the results are
the normal library's bit for bit."""
import os
import subprocess
import sys
import textwrap

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_CHILD = textwrap.dedent("""
    import sys, torch
    sys.path.insert(0, {root!r})
    from paper_2512_21571_b200 import binding as nnc
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    randn = lambda *shape, dtype=torch.float32: torch.randn(*shape, generator=g, device="cuda").to(dtype)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    BF16, F16, F32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
    out = {{}}
    for tokens, heads, d, rot in ((1, 1, 64, 64), (1, 40, 128, 128), (2003, 24, 96, 48), (5, 2, 66, 66), (301, 3, 9, 2), (33, 70, 192, 64), (2, 2, 1024, 1024)):
        for dtype in (BF16, F32):
            for inter in (False, True):
                x, pos = randn(tokens, heads, d, dtype=dtype), torch.arange(tokens, device="cuda", dtype=torch.int32) * 7 - 3
                freq, _ = nnc.rope_frequencies(rot)
                y = nnc.op_rope(x, pos, freq, interleaved=inter)
                nnc.op_rope(y, pos, freq, interleaved=inter, inverse=True, out=y)
                out[f"rope{{tokens}}.{{heads}}.{{d}}.{{rot}}.{{dtype}}.{{inter}}"] = [y.cpu()]
    scratch = nnc.attn_paged_scratch()
    for kv, dtype in ((BF16, BF16), (BF16, F32), (F16, F16), (F16, F32), (E4M3, BF16), (E4M3, F16), (E4M3, F32)):
        for lens, page, heads, group, d, window in (([0, 1, 17, 700], 16, 2, 4, 128, 0), ([30011], 64, 1, 16, 64, 0), ([70, 5000, 129], 256, 2, 17, 128, 99),
                                                    ([33] * 300, 32, 2, 2, 64, 0), ([131072], 256, 1, 40, 64, 0)):
            used = [-(-n // page) for n in lens]
            cache = nnc.PagedKV.empty(sum(used) + 1, page, heads, d, kv, len(lens), max(used))
            at = 1
            for b, n in enumerate(used):
                cache.page_table[b, :n] = torch.arange(at, at + n, device="cuda")
                at += n
            pos, seq = ints([i for n in lens for i in range(n)]), ints([b for b, n in enumerate(lens) for _ in range(n)])
            k, v = (randn(len(pos), heads, d, dtype=dtype) for _ in range(2))
            if kv is not E4M3:
                v[len(pos) // 2, 0, 5] = float("inf")
            nnc.op_kv_write_paged(cache, k, v, pos, seq)
            q = randn(len(lens), heads * group, d, dtype=dtype)
            got = nnc.op_attn_decode_paged(q, cache, ints(lens), window=window, scratch=scratch, want_lse=True)
            rows = nnc.op_kv_read_paged(cache, pos[-2000:], seq[-2000:], dtype=F32)
            out[f"{{kv}}.{{dtype}}.{{len(lens)}}.{{page}}.{{group}}"] = [t.cpu() for t in (*got, *rows)]
            assert nnc.op_status() == 0
            cache.page_table[0, 0] = 1 << 30                      # what no address check of the kernels' own lets through
            nnc.op_attn_decode_paged(q, cache, ints(lens), scratch=scratch)
            nnc.op_kv_read_paged(cache, pos[-1:] + (1 << 20), seq[-1:])
            assert nnc.op_status() == 0x100
    torch.cuda.synchronize()
    torch.save({{"out": out, "report": nnc.bounds_check_report()}}, sys.argv[1])
""")


@pytest.mark.gpu
def test_paged_operations_run_clean_in_the_checked_build(tmp_path):
    import torch
    from paper_2512_21571_b200 import build
    build.build()
    prog = tmp_path / "child.py"
    prog.write_text(_CHILD.format(root=ROOT))
    results = {}
    for tag, lib in (("normal", None), ("checked", build.build(checked=True))):
        env = {k: v for k, v in os.environ.items() if k != "NNC_LIBRARY"}
        if lib:
            env["NNC_LIBRARY"] = lib
        res = tmp_path / (tag + ".pt")
        r = subprocess.run([sys.executable, str(prog), str(res)], capture_output=True, text=True, timeout=900, env=env)
        assert r.returncode == 0, r.stdout + r.stderr
        results[tag] = torch.load(res)
    assert results["normal"]["report"] == (-1, 0)
    assert results["checked"]["report"] == (0, 0), "the checked build counted out-of-range indices"
    for key, tensors in results["normal"]["out"].items():
        for a, b in zip(tensors, results["checked"]["out"][key]):
            assert torch.equal(a.nan_to_num(nan=1e30), b.nan_to_num(nan=1e30)), key


def test_every_kernel_of_the_paged_operations_has_checks():
    """Their sources name the bounds-check macro; codes are their own."""
    import re
    seen = {}
    for name in sorted(f for f in os.listdir(os.path.join(ROOT, "paper_2512_21571_b200", "csrc")) if f.endswith((".cu", ".cuh"))):
        text = open(os.path.join(ROOT, "paper_2512_21571_b200", "csrc", name)).read()
        for code in re.findall(r"NNC_BC\((?:[^;]*?),\s*(\d+)\)", text):
            assert seen.setdefault(code, name) == name, code
    assert {"attn_paged.cu", "kv_paged.cu", "rope.cu"} <= set(seen.values())
