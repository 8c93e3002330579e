"""Workgroups of attention to short sequences, of which no item is cut: one for each item as far as they run at a time, on devices that need not be there."""
from recording_runtime import record

SCRIPT = r"""
import ctypes as C
def grid(count, new, length, heads, kv_heads, dim, cus=256, window=0):
    device(cus, 1)
    ctx = sb.Context(0, 0)
    A = fake(1)
    rows = kv_heads * 64
    cache = sb.KvCache(A, A, A, A, 5000, rows * dim // 2, rows * sb.mx_scale_pitch(dim), 64, kv_heads, dim)
    seqs = sb.Sequences(A, A, A, 1000, count, 1000, new, length)
    need = sb.load().sbits_kv_attention_ws_bytes(ctx.h, C.addressof(cache), C.addressof(seqs), count * new, heads)
    log()
    rc = sb.load().sbits_kv_attention(ctx.h, C.addressof(cache), C.addressof(seqs), count * new, heads, A, heads * dim, dim, 0.1, 1, window, A, heads * dim, dim, None, fake(need), need)
    assert rc == 0
    lines = [x.split() for x in log() if x.startswith("launch")]
    return need, ["few" in x[1] for x in lines], int(lines[0][3].split(",")[0])
answer([grid(*a) for a in %r])
"""


def test_a_workgroup_for_each_short_item(tmp_path):
    cases = [((1, 8, 9, 16, 2, 256), 8),           # four tiles of rows on two heads
             ((1, 1, 64, 4, 4, 64), 4), ((10, 1, 154, 16, 4, 128), 40), ((108, 1, 29, 112, 16, 128), 512), ((108, 1, 29, 112, 16, 256), 256), ((108, 1, 29, 112, 16, 128, 32), 64),
             ((1, 1, 1000, 32, 8, 128), 16)]
    for (case, want), (need, few, grid) in zip(cases, record(tmp_path, SCRIPT % [c for c, _ in cases])):
        assert need == 0 and few == [True] and grid == want, (case, grid)


def test_a_short_window_leaves_no_item_to_cut(tmp_path):
    cases = [((21, 5, 60000, 7, 1, 128, 256, 78), True), ((21, 5, 60000, 7, 1, 128, 256, 891), True), ((21, 5, 60000, 7, 1, 128, 256, 892), False), ((21, 5, 60000, 7, 1, 128), False)]
    for (case, short), (need, few, grid) in zip(cases, record(tmp_path, SCRIPT % [c for c, _ in cases])):
        assert need > 0 and few == ([True] if short else [True, False]) and grid == 512, (case, grid)
