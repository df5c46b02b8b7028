"""Page bounds, scores, selection, attention over selected pages and behind shared prefixes through the bounds-checked debugging build: no
index misses its extent, and the results are the normal library's bit for bit."""
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
    scratch = nnc.attn_paged_scratch()
    for kv, dtype in ((BF16, BF16), (BF16, F32), (F16, F16), (F16, F32), (E4M3, BF16), (E4M3, F16), (E4M3, F32)):
        # sequences of one batch share their first `common` positions
        for lens, common, page, heads, group, d, n in (([0, 1, 17, 700], 0, 16, 2, 4, 128, 5), ([5000, 4099, 4096, 5001, 4500, 70], 4096, 64, 1, 16, 64, 9),
                                                       ([2600, 2570, 2561], 2560, 256, 2, 17, 128, 3), ([330] * 150, 320, 32, 2, 3, 64, 40)):
            whole = common // page
            own = [max(0, -(-x // page) - whole) for x in lens]
            columns = max(whole + x for x in own) + 1
            columns = max(columns, 150_000_000 // (2 * len(lens) * page * heads * d))     # wide: the prefix is read once
            cache = nnc.PagedKV.empty(whole + sum(own) + 1, page, heads, d, kv, len(lens), columns)
            at = whole + 1
            for b, x in enumerate(own):
                cache.page_table[b, :whole] = torch.arange(1, whole + 1, device="cuda")
                cache.page_table[b, whole:whole + x] = torch.arange(at, at + x, device="cuda")
                at += x
            tokens = [(i, 0) for i in range(common)] + [(i, b) for b, x in enumerate(lens) for i in range(common, x)]
            pos, seq = ints([t[0] for t in tokens]), ints([t[1] for t in tokens])
            k, v = (randn(len(tokens), heads, d, dtype=dtype) for _ in range(2))
            if kv is not E4M3:
                v[len(tokens) // 2, 0, 5] = float("inf")
            nnc.op_kv_write_paged(cache, k, v, pos, seq)
            q, ends = randn(len(lens), heads * group, d, dtype=dtype), ints(lens)
            starts, shared = ints([0, len(lens) - 1, len(lens)]), ints([common, 0])

            def step():
                bounds = nnc.op_page_bounds(cache, nnc.page_bounds(cache), ends)
                nnc.op_page_bounds(cache, bounds, ends, torch.clamp(ends - 1, min=0))
                scores = nnc.op_score_pages(q, cache, bounds, ends)
                held = torch.arange(columns, device="cuda").view(1, 1, -1) * page < ends.view(-1, 1, 1)
                pages, counts = nnc.op_select_pages(scores, ends, page, n)
                return [bounds, torch.where(held, scores, 0), counts, torch.where(torch.arange(n, device="cuda") < counts.unsqueeze(2), pages, 0),
                        *nnc.op_attn_selected_paged(q, cache, ends, pages, counts, scratch=scratch, want_lse=True),
                        *nnc.op_attn_prefix_paged(q, cache, ends, starts, shared, want_lse=True)]
            out[f"{{kv}}.{{dtype}}.{{len(lens)}}.{{page}}.{{group}}"] = [t.cpu() for t in step()]
            assert nnc.op_status() == 0
            cache.page_table[0, 0] = 1 << 30                      # what no address check of the kernels' own lets through
            cache.page_table[-1, 0] = -5
            step()
            assert nnc.op_status() == 0x100
            pages, counts = torch.full((len(lens), heads, n), 1 << 30, dtype=torch.int32, device="cuda"), torch.full((len(lens), heads), n + 9, dtype=torch.int32, device="cuda")
            nnc.op_attn_selected_paged(q, cache, ends, pages, counts, scratch=scratch)
            nnc.op_attn_prefix_paged(q, cache, ends + (1 << 28), ints([5, -7, 1 << 30]), ints([1 << 30, -1]))
            assert nnc.op_status() == 0x100
    for rows, columns, n in ((1, 1, 2), (3, 257, 64), (2, 2049, 100), (1, 131072, 4096), (300, 33, 33)):
        scores = randn(rows, 2, columns).round(decimals=1)
        out[f"select{{rows}}.{{columns}}"] = [t.cpu() for t in nnc.op_select_pages(scores, ints([columns * 16 - 3] * rows), 16, n)]
    torch.cuda.synchronize()
    torch.save({{"out": out, "report": nnc.bounds_check_report()}}, sys.argv[1])
""")


@pytest.mark.gpu
def test_page_operations_run_clean_in_the_checked_build(tmp_path):
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
            assert torch.equal(a.float().nan_to_num(nan=1e30), b.float().nan_to_num(nan=1e30)), key


def test_every_kernel_of_the_page_operations_has_checks():
    csrc = os.path.join(ROOT, "paper_2512_21571_b200", "csrc")
    for name in ("pages.cu", "attn_selected.cu", "attn_prefix.cu", "attn_prefix_tail.cu", "attn_paged_body.cuh"):
        assert "NNC_BC(" in open(os.path.join(csrc, name)).read(), name
