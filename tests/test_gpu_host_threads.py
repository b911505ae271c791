"""First calls of the operators from many host threads at once: what they set up once per
device is set up when the first of them launches."""
import subprocess
import sys
import textwrap

import pytest

from tests.conftest import ROOT
from tests.helpers import ensure_lib

pytestmark = pytest.mark.gpu


def test_first_calls_from_many_threads():
    ensure_lib()
    code = textwrap.dedent("""
        import threading
        import torch
        from paper_2606_31160_gb300 import sd
        sd.lib()
        torch.manual_seed(0)
        B, H, n, D, keep, T = 1, 2, 6000, 128, 500, 12
        k = torch.randn((B, H, n, D), device="cuda").to(torch.bfloat16)
        src = sd.KVCache(k, k.clone(), torch.full((B,), n, dtype=torch.int32, device="cuda"))
        w = torch.rand((B, H, n), device="cuda")
        q = torch.randn((B, 4, 8, D), device="cuda").to(torch.bfloat16)
        c8 = [sd.KV8Cache.empty(B, H, n, D) for _ in range(T)]
        dst = [sd.KVCache.empty(B, H, keep, D) for _ in range(T)]
        torch.cuda.synchronize()
        out, errors, gate = [None] * T, [], threading.Barrier(T)

        def work(i):
            try:
                s = torch.cuda.Stream()
                with torch.cuda.stream(s):
                    gate.wait()
                    sd.kv_evict(src, w, dst[i], keep)
                    sd.kv8_store(c8[i], src)
                    out[i] = (dst[i].k, sd.kv8_attention(q, c8[i]), sd.attention_weights(q, src))
                s.synchronize()
            except Exception as e:
                errors.append(repr(e))

        threads = [threading.Thread(target=work, args=(i,)) for i in range(T)]
        [t.start() for t in threads]
        [t.join() for t in threads]
        torch.cuda.synchronize()
        assert not errors, errors
        want = torch.sort(torch.topk(w, keep, dim=-1).indices, dim=-1).values
        assert torch.equal(out[0][0], k.gather(2, want[..., None].expand(-1, -1, -1, D)))
        for o in out[1:]:
            assert all(torch.equal(a, b) for a, b in zip(o, out[0]))
        assert sd.get_device_error() == 0
        print("ok")
    """)
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stderr[-2000:]
