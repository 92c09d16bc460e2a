"""tkv_prompt_attn against float64: lengths from none to several tiles, packed, padded and chunked sequences, head
groups, types, strides, rows without keys, what lies behind the sequences, streams and replayed graphs.

Tolerance: with u = half a step of the type (fp16 2^-11, bf16 2^-8), a weight is rounded once (u, relative), the output once
(u, relative), the sums and logits are float32 (products of 16-bit numbers are exact there): |o - ref| <= u |ref| + 1.1 u sum_j w_j
|v_j|, w the exact weights.  The logarithm of the sum: 1e-5 absolute (float32 logits of magnitude up to 32: 128 terms, 2^-24 each)."""
import numpy as np
import pytest
import torch

import paper_2505_19586_amd as tkv
from oracle.prompt import prompt_attention

pytestmark = pytest.mark.gpu
SM = 128 ** -0.5
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def _rows(n, heads, dtype, seed, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (gain * torch.randn(n, heads, 128, generator=g, device="cuda")).to(dtype)


def _np(x):
    return x.double().cpu().numpy()


def _compare(out, lse, q, k, v, causal, dtype, sm=SM):
    """One sequence; q the last tokens of k, v."""
    q, k, v = _np(q), _np(k), _np(v)
    ref, ref_lse = prompt_attention(q, k, v, sm, causal)
    size, _ = prompt_attention(q, k, np.abs(v), sm, causal)
    u = HALF_STEP[dtype]
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    err = np.abs(_np(out) - ref)
    assert (err <= u * np.abs(ref) + 1.1 * u * size + tiny).all(), float((err / (u * size + 1e-30)).max())
    if lse is not None:
        lse = _np(lse)
        assert np.array_equal(np.isneginf(lse), np.isneginf(ref_lse))
        seen = np.isfinite(ref_lse)
        assert np.abs(lse[seen] - ref_lse[seen]).max(initial=0.0) <= 1e-5


def _run(q_lens, k_lens, hq, hkv, dtype, causal=True, seed=0, some=None):
    q, k, v = _rows(sum(q_lens), hq, dtype, seed), _rows(sum(k_lens), hkv, dtype, seed + 1), _rows(sum(k_lens), hkv, dtype, seed + 2)
    plan = tkv.PromptAttention(n_q_heads=hq, n_kv_heads=hkv, dtype=dtype, causal=causal, batch=len(q_lens))
    out, lse = plan.attend(q, k, v, SM, q_lens, k_lens, lse=True)
    torch.cuda.synchronize()
    q0 = k0 = 0
    for nq, nk in zip(q_lens, k_lens):
        at = slice(q0, q0 + nq)
        _compare(out[at], lse[at], q[at], k[k0:k0 + nk], v[k0:k0 + nk], causal, dtype)
        q0, k0 = q0 + nq, k0 + nk


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 517])
def test_whole_prompts(n, dtype):
    print(f"case prompt n={n} {dtype}", flush=True)
    _run([n], [n], 8, 2, dtype, seed=n)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 5), (14, 2), (8, 1), (16, 1), (33, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_head_groups(hq, hkv, causal):
    print(f"case heads {hq}/{hkv} causal={causal}", flush=True)
    _run([77], [150], hq, hkv, torch.float16, causal, seed=hq)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_packed_sequences_chunks_and_empty_ones(causal, dtype):
    print(f"case packed causal={causal} {dtype}", flush=True)
    _run([1, 0, 130, 5, 64, 1, 40], [1, 70, 130, 300, 64, 515, 0], 8, 2, dtype, causal, seed=3)


def test_tokens_ahead_of_every_key_yield_zeros():
    """More query tokens than keys: the first see none."""
    print("case more queries than keys", flush=True)
    _run([100, 9], [37, 3], 4, 2, torch.float16, seed=5)


@pytest.mark.parametrize("nq,nk", [(1, 1000), (1, 5003), (3, 2500), (17, 4100), (200, 1500)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_few_rows_over_many_keys(nq, nk, dtype):
    print(f"case few rows {nq} over {nk} {dtype}", flush=True)
    _run([nq], [nk], 8, 2, dtype, seed=nk)


def test_single_tokens_of_a_batch_of_64():
    lens = [(37 * b) % 300 for b in range(64)]
    print("case 64 single tokens", flush=True)
    _run([1] * 64, lens, 4, 1, torch.float16, seed=9)


def test_padded_batch_slices_and_untouched_rows():
    """Sequences in a padded batch of fused rows [B][n][Hq + 2 Hkv][128]; rows behind the sequences hold NaN in k and v and
    stay as they were in out and lse."""
    print("case padded batch", flush=True)
    b, n, hq, hkv, lens = 4, 150, 8, 2, [150, 1, 97, 64]
    rows = _rows(b * n, hq + 2 * hkv, torch.float16, 11)
    for i, m in enumerate(lens):
        rows[i * n + m:(i + 1) * n] = float("nan")
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    out = torch.full((b * n, hq + 1, 128), 7.0, dtype=torch.float16, device="cuda")[:, :hq]   # a wider row's slice
    lse = torch.full((b * n, hq), 5.0, device="cuda")
    plan = tkv.PromptAttention(n_q_heads=hq, n_kv_heads=hkv, batch=b)
    starts = [i * n for i in range(b)]
    plan.attend(q, k, v, SM, lens, q_starts=starts, k_starts=starts, out=out, lse=lse)
    torch.cuda.synchronize()
    for i, m in enumerate(lens):
        at = slice(i * n, i * n + m)
        _compare(out[at], lse[at], q[at], k[at], v[at], True, torch.float16)
        assert (out[i * n + m:(i + 1) * n] == 7).all() and (lse[i * n + m:(i + 1) * n] == 5).all()


def test_heads_outermost_and_sequences_in_any_order():
    print("case heads outermost", flush=True)
    q, k, v = (_rows(300, h, torch.bfloat16, 20 + h).transpose(0, 1).contiguous().transpose(0, 1) for h in (6, 2, 2))
    plan = tkv.PromptAttention(n_q_heads=6, n_kv_heads=2, dtype=torch.bfloat16, batch=2)
    out = torch.zeros(6, 300, 128, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    plan.attend(q, k, v, SM, [100, 70], [200, 100], q_starts=[200, 10], k_starts=[0, 200], out=out)
    torch.cuda.synchronize()
    _compare(out[200:300], None, q[200:300], k[:200], v[:200], True, torch.bfloat16)
    _compare(out[10:80], None, q[10:80], k[200:], v[200:], True, torch.bfloat16)
    assert (out[:10] == 0).all() and (out[80:200] == 0).all()


def test_one_dominant_key_and_large_logits():
    """Logits up to hundreds, the running maximum far behind in the last tile; equal keys give equal weights."""
    print("case dominant keys", flush=True)
    n = 400
    q, k, v = _rows(n, 4, torch.float16, 30, 4.0), _rows(n, 1, torch.float16, 31, 4.0), _rows(n, 1, torch.float16, 32)
    k[390] = 3 * q[395, 0]
    k[5:200] = k[4]
    plan = tkv.PromptAttention(n_q_heads=4, n_kv_heads=1)
    out = plan.attend(q, k, v, SM, [n])
    torch.cuda.synchronize()
    # logits of magnitude L carry an error of 2^-24 128 L / sqrt(128) at most in float32, relative in the weights
    ref, _ = prompt_attention(_np(q), _np(k), _np(v), SM)
    size, _ = prompt_attention(_np(q), _np(k), np.abs(_np(v)), SM)
    top = float(np.abs(np.einsum("qhd,kd->qhk", _np(q), _np(k)[:, 0])).max() * SM)
    assert (np.abs(_np(out) - ref) <= 2.0 ** -11 * np.abs(ref) + (1.1 * 2.0 ** -11 + 2.0 ** -19 * top) * size + 2.0 ** -25).all()


def test_keys_seen_by_nobody_do_not_matter():
    """Rows behind k_len and the other sequence's rows may hold anything, within the same tile too."""
    print("case other rows", flush=True)
    q, k, v = _rows(90, 8, torch.float16, 40), _rows(90, 2, torch.float16, 41), _rows(90, 2, torch.float16, 42)
    plan = tkv.PromptAttention(n_q_heads=8, n_kv_heads=2)
    want = plan.attend(q[:50], k[:50], v[:50], SM, [50]).clone()
    k[50:], v[50:] = float("nan"), float("inf")
    got = plan.attend(q[:50], k, v, SM, [50])
    assert torch.equal(want, got)


def test_side_stream_replayed_graph_and_shared_workspace():
    print("case graph", flush=True)
    q, k, v = _rows(3, 8, torch.float16, 50), _rows(2000, 2, torch.float16, 51), _rows(2000, 2, torch.float16, 52)
    plan = tkv.PromptAttention(n_q_heads=8, n_kv_heads=2)
    want = plan.attend(q, k, v, SM, [3], [2000]).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = plan.attend(q, k, v, SM, [3], [2000])
    torch.cuda.synchronize()
    assert torch.equal(want, got)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.graph(graph):
        plan.attend(q, k, v, SM, [3], [2000], out=out)
    for _ in range(4):
        plan.workspace.fill_(0xFF)          # whatever it held
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, plan.attend(q, k, v, SM, [3], [2000]))
        q += 0.25


def test_stream_argument_orders_new_outputs():
    """New outputs are made on the stream that writes them, whatever the current one is busy with."""
    print("case stream argument", flush=True)
    q, k, v = _rows(40, 8, torch.float16, 53), _rows(40, 2, torch.float16, 54), _rows(40, 2, torch.float16, 55)
    plan = tkv.PromptAttention(n_q_heads=8, n_kv_heads=2)
    want, want_lse = plan.attend(q, k, v, SM, [33], [33], lse=True)
    side, busy = torch.cuda.Stream(), torch.zeros(1 << 28, device="cuda")
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        for _ in range(20):
            busy += 1
        got, lse = plan.attend(q, k, v, SM, [33], [33], lse=True, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(want, got) and torch.equal(want_lse, lse) and not got[33:].any()


def test_sequences_that_share_keys_in_any_order():
    print("case shared keys", flush=True)
    q, k, v = _rows(90, 8, torch.float16, 56), _rows(200, 2, torch.float16, 57), _rows(200, 2, torch.float16, 58)
    plan = tkv.PromptAttention(n_q_heads=8, n_kv_heads=2, batch=3)
    out = plan.attend(q, k, v, SM, [30, 0, 50], [200, 7, 150], q_starts=[60, 10, 0], k_starts=[0, 0, 50])
    _compare(out[60:], None, q[60:], k, v, True, torch.float16)
    _compare(out[:50], None, q[:50], k[50:], v[50:], True, torch.float16)
    assert not out[50:60].any()
    with pytest.raises(tkv.TkvError):
        plan.attend(q, k, v, SM, [30, 0, 50], [200, 7, 150], q_starts=[49, 10, 0], k_starts=[0, 0, 50])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("q_lens,k_lens", [([256], [3000]), ([300, 1, 20], [5000, 700, 20]), ([1, 8], [9000, 40]), ([2], [70000])])
def test_split_keys(q_lens, k_lens, dtype):
    """Both kernels with their keys in pieces, joined by a wave per row and (more than 16 pieces) by a workgroup."""
    print(f"case split {q_lens} {k_lens} {dtype}", flush=True)
    _run(q_lens, k_lens, 8, 2, dtype, seed=sum(q_lens))


@pytest.mark.parametrize("q_lens,k_lens", [([1] * 40, [7000] + [90] * 39), ([1] * 63 + [8], [5] * 62 + [0, 30000]),
                                           ([9] + [1] * 35 + [0], [9000] + [200] * 35 + [50]), ([40] * 40 + [70], [40] * 40 + [12000])])
def test_long_sequences_among_many(q_lens, k_lens):
    """More row tiles than compute units (8 KV heads), one sequence far above the even share: that one is split."""
    print(f"case ragged {len(q_lens)} sequences, {max(k_lens)} keys", flush=True)
    _run(q_lens, k_lens, 16, 8, torch.float16, seed=len(q_lens))


def test_stream_with_compute_unit_mask():
    """On part of the machine the keys are split into fewer pieces."""
    import ctypes as C
    print("case masked stream", flush=True)
    hip = C.CDLL("libamdhip64.so")
    create = hip.hipExtStreamCreateWithCUMask
    create.argtypes = [C.POINTER(C.c_void_p), C.c_uint32, C.POINTER(C.c_uint32)]
    create.restype = C.c_int
    mask = (C.c_uint32 * 8)(0xFFFF0000, 0xFFFFFFFF, 0xFFFFFFFF, 0x0000FFFF, 0, 0, 0, 0)   # 96 units
    handle = C.c_void_p()
    if create(C.byref(handle), 8, mask) != 0 or not handle.value:
        pytest.skip("streams with a compute-unit mask are not available")
    try:
        q, k, v = _rows(70, 8, torch.float16, 63), _rows(6000, 2, torch.float16, 64), _rows(6000, 2, torch.float16, 65)
        plan = tkv.PromptAttention(n_q_heads=8, n_kv_heads=2)
        torch.cuda.synchronize()
        for n in (70, 3):
            out = torch.empty_like(q[:n])
            torch.cuda.synchronize()
            plan.attend(q[:n], k, v, SM, [n], [6000], out=out, stream=torch.cuda.ExternalStream(handle.value))
            torch.cuda.synchronize()
            _compare(out, None, q[:n], k, v, True, torch.float16)
    finally:
        torch.cuda.synchronize()
        hip.hipStreamDestroy.argtypes = [C.c_void_p]
        hip.hipStreamDestroy(handle)


def test_large_offsets():
    """Sequences that begin beyond 2^31 elements of a tensor."""
    print("case large offsets", flush=True)
    n = (1 << 31) // 128 + 300              # rows of 1 head: more than 2^31 elements
    k = torch.zeros(n, 1, 128, dtype=torch.float16, device="cuda")
    v = torch.zeros(n, 1, 128, dtype=torch.float16, device="cuda")
    q, kk, vv = _rows(20, 2, torch.float16, 60), _rows(200, 1, torch.float16, 61), _rows(200, 1, torch.float16, 62)
    k[-200:], v[-200:] = kk, vv
    plan = tkv.PromptAttention(n_q_heads=2, n_kv_heads=1)
    out = plan.attend(q, k, v, SM, [20], [200], q_starts=[0], k_starts=[n - 200])
    torch.cuda.synchronize()
    _compare(out, None, q, kk, vv, True, torch.float16)


def test_long_context_against_a_float32_reference():
    """65536 keys: every row against float64 sums on the GPU."""
    print("case 65536 keys", flush=True)
    nq, nk = 37, 65536
    q, k, v = _rows(nq, 8, torch.float16, 70), _rows(nk, 2, torch.float16, 71), _rows(nk, 2, torch.float16, 72)
    plan = tkv.PromptAttention(n_q_heads=8, n_kv_heads=2)
    out, lse = plan.attend(q, k, v, SM, [nq], [nk], lse=True)
    hidden = torch.ones(nq, nk, dtype=torch.bool, device="cuda").triu(nk - nq + 1)
    for h in range(8):
        s = (q[:, h].double() @ k[:, h // 4].double().T.contiguous() * SM).masked_fill(hidden, -float("inf"))
        w = torch.softmax(s, 1)
        ref, size = w @ v[:, h // 4].double(), w @ v[:, h // 4].double().abs()
        u = 2.0 ** -11
        assert ((out[:, h].double() - ref).abs() <= u * ref.abs() + 1.1 * u * size + 2.0 ** -25).all()
        assert (lse[:, h].double() - torch.logsumexp(s, 1)).abs().max() <= 1e-5
