"""Paged decoding steps that pass their own longest length in a workspace sized once, for the capacity: every
step is taken, writes nothing behind the workspace and gives the oracle's rows (tolerances of test_paged_gpu)."""
import pytest
import torch

import guards
import paging
from paper_2607_08186_gb300 import binding, build, inputs
from test_paged_gpu import I32, _assert_rows, _case, _i32

pytestmark = pytest.mark.gpu

CROSS, LOCAL = inputs.CROSS, inputs.LOCAL


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


# lengths whose plans have more splits than the capacity's among them
@pytest.mark.parametrize("B,n,Hq,Hkv,Dh,P,steps", [(1, 4, 32, 8, 128, 16, (608, 1200, 1216, 1792, 1808, 64, 1, 2048)),
                                                   (3, 4, 24, 2, 256, 16, (200, 416, 608, 1999, 2048)),
                                                   (2, 4, 96, 8, 128, 8, (250, 800, 1111, 2048)),
                                                   (4, 8, 16, 4, 64, 5, (77, 304, 912, 2048))])
def test_one_workspace_for_every_step(B, n, Hq, Hkv, Dh, P, steps):
    cap = 2048
    width = -(-cap // P)
    q, kc, vc = _case(B, cap, n, Hq, Hkv, Dh, 5)
    kp, table = paging.to_pages(kc, [cap] * B, P, n, 1, width=width)
    vp, _ = paging.to_pages(vc, [cap] * B, P, n, 1, width=width)
    kd, vd, td, qd = kp.cuda(), vp.cuda(), table.cuda(), q.cuda()
    ws = guards.empty((binding.sfa_decode_paged_workspace_bytes(B, cap, n, Hq, Hkv, Dh, LOCAL, cap * n),), torch.uint8, 0xFF,
                      what="workspace")
    st = torch.zeros(1, dtype=I32, device="cuda")
    for T in steps:
        lens = [max(1, T - 50 * b) for b in range(B)]
        for mode, w in ((CROSS, 0), (LOCAL, 300)):
            o, lse = guards.empty(q.shape, torch.bfloat16, 7.0), guards.empty((B, Hq, n), torch.float32, 7.0)
            binding.sfa_decode_paged(qd, kd, vd, td, _i32(lens).cuda(), o, n, mode, ws, max_tokens=T, lse=lse, window=w,
                                     dev_status=st)
            assert int(st.item()) == 0
            for b, t in enumerate(lens):
                _assert_rows(o.cpu(), lse.cpu(), q, kc[:, :t * n], vc[:, :t * n], t, b, n, mode, w)
    with pytest.raises(binding.HdError):  # a workspace that is too small is refused as ever
        binding.sfa_decode_paged(qd, kd, vd, td, _i32([1] * B).cuda(), o, n, CROSS, ws[:-1 - ws.numel() // 2], max_tokens=cap)
