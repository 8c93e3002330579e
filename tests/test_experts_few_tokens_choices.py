"""Which routing kernels the tests of layers for few tokens run."""
from recording_runtime import record
from test_gpu_experts_few_tokens import ROUTERS, TOKENS

SCRIPT = r"""
import ctypes as C
ctx = sb.Context(0, 0)
out = []
hidden, inner = 64, 32
for at, router in enumerate(%r):
    for tokens in %r:
        for kind in (0, 1):
            r = sb.Router(**router)
            up = sb.Mx(fake(1 << 20), fake(1 << 20), r.experts * 2 * inner, hidden, hidden // 2, 4)
            down = sb.Mx(fake(1 << 20), fake(1 << 20), r.experts * hidden, inner, inner // 2, 4)
            need = ctx.expert_layer_ws_bytes(r, tokens, up, down)
            log()
            rc = sb.load().sbits_expert_layer(ctx.h, C.addressof(r), fake(1 << 20), kind, r.experts, None, fake(1 << 20), hidden, tokens, C.addressof(up),
                                              C.addressof(down), fake(1 << 20), hidden, fake(1 << 20), fake(1 << 20), 0, fake(need), need)
            out.append([at, tokens, kind, rc, [line.split()[1] for line in log() if line.startswith("launch")]])
answer(out)
"""


def test_layers_of_few_tokens_run_the_kernels_that_their_tests_are_for(tmp_path):
    for at, tokens, kind, rc, names in record(tmp_path, SCRIPT % ([k[0] for k in ROUTERS], TOKENS)):
        registers = ROUTERS[at][1]
        one = tokens <= 8 and registers is not None
        assert rc == 0 and ("route_and_list_kernel" in names[0]) == one and len(names) == (4 if one else 5), names
        if one:
            assert "route_and_list_kernelILb%dELi%dE" % (kind, registers) in names[0]
        else:
            assert "route_kernelILb%dE" % kind in names[0] and "expert_lists_kernel" in names[1]
