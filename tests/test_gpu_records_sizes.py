"""Single tokens over quantised records of very different size: what a record holds, or how large it is, must not cost the
records that a token attends.  The bounds are those of the attended values, not of the largest value in the pool.

For key j with weight p_j and value v_j, and a score that is off by at most
  d_j = (2^-23 (D / 16 + 4) sum_i |q_i k_ji| + 2^-22 max |q| sum_i |k_ji|) |scale|
(fp32 sums of D / 16 steps and the scaling; the query's two e4m3 terms), an output number is off by at most
  * 4 sum_j p_j d_j (|v_j| + |out|): a weight moves by a factor of at most e^(2 d_j), and the normaliser with it;
  * (2^-11 + 2^-23 (K / 16 + 64)) sum_j p_j |v_j|: the weights' rounding to f16 and the fp32 sums of K / 16 steps;
  * 2 K 2^-(20 + lift) M, M = max_j p_j max |v_j over the group of 128|: a weight's three e4m3 terms are off by 2^-20 of the unit in
    which the largest weight times scale lies above 2^lift, a code is at most 448 and the group's largest one above 224;
    2048 2^lift >= K, so this is at most 2^-8 M;
  * 2^-8 |out|: the rounding of out to bf16.
"""
import numpy as np
import pytest
import torch

import paper_2608_07009_b200 as hs
from oracle import record_oracle as ro
from test_gpu_records import DEV, bf16, chunk_case, numbers, run_chunk

pytestmark = pytest.mark.gpu


def exact_bf16(x):
    return ro.bf16_values(ro.round_to_bf16(x))


def attended(num, q, Dv, scale, D):
    """One request: num [K][D] of the keys that are there, q [H][D].  (out, lse, bound of out, bound of lse)."""
    K = len(num)
    out, lse = ro.attention(num, np.ones(K, bool), q, Dv, scale)
    p = np.exp(scale * (q @ num.T) - lse[:, None])
    d = (2.0 ** -23 * (D / 16 + 4) * (np.abs(q) @ np.abs(num).T)
         + 2.0 ** -22 * np.abs(q).max(1)[:, None] * np.abs(num).sum(1)[None]) * abs(scale)
    v = np.abs(num[:, :Dv])
    lift = 0
    while lift < 6 and K > 2048 << lift:
        lift += 1
    m = (p[:, :, None] * v.reshape(K, -1, 128).max(2)[None]).max(1).repeat(128, axis=1)
    bound = (4 * ((p * d) @ v + (p * d).sum(1)[:, None] * np.abs(out)) + (2.0 ** -11 + 2.0 ** -23 * (K / 16 + 64)) * (p @ v)
             + 2 * K * 2.0 ** -(20 + lift) * m + 2.0 ** -8 * np.abs(out))
    return out, lse, bound, 2 * (p * d).sum(1) + 2.0 ** -20 * np.maximum(1, np.abs(lse))


def hold(out, lse, num, table, q, Dv, scale, D):
    out, lse = numbers(out), numbers(lse)
    for n in range(len(q)):
        here = table[n][table[n] >= 0]
        o, s, bo, bs = attended(num[here], q[n], Dv, scale, D)
        worst = np.max(np.abs(out[n] - o) / np.maximum(bo, 1e-300))
        assert worst <= 1, (n, worst)
        assert np.all(np.abs(lse[n] - s) <= bs), n


def slot_table(raw, table, q, D, Dq, Dv, scale):
    return hs.record_attention(hs.RecordFormat(D, Dq), torch.from_numpy(raw).to(DEV), torch.from_numpy(table).to(DEV), bf16(q).to(DEV), Dv, scale)


# one block a request, blocks that merge in a cluster, blocks that merge through a workspace
SHAPES = [(1, 128), (3, 77), (16, 1000), (1, 2048), (33, 700)]


@pytest.mark.parametrize("size", [1e-2, 1e-3, 1e-4, 300.0])
@pytest.mark.parametrize("N,K", SHAPES)
@pytest.mark.parametrize("D,Dq,Dv,H", [(144, 128, 128, 16), (576, 512, 512, 16), (144, 128, 128, 40), (320, 256, 256, 24)])
def test_zero_records_and_zero_groups_cost_the_others_nothing(size, N, K, D, Dq, Dv, H):
    rng = np.random.default_rng(K + D)
    x = rng.standard_normal((K, D)) * size
    x[5] = 0                                                      # a padded token
    x[40, :128] = 0                                               # a group of zeros
    x[41, :128] = -0.0
    if Dq > 128:
        x[70, 128:Dq] = 0
    raw = ro.encode(exact_bf16(x), Dq)
    num = ro.decode(raw, D, Dq)
    table = np.stack([rng.permutation(K) for _ in range(N)]).astype(np.int32)
    table[0, ::7] = np.where(np.isin(table[0, ::7], (5, 40, 41, 70)), table[0, ::7], -1)
    q = exact_bf16(rng.standard_normal((N, H, D)) * (0.05 / size if size < 1 else 2e-4))
    out, lse = slot_table(raw, table, q, D, Dq, Dv, 1.0)
    hold(out, lse, num, table, q, Dv, 1.0, D)


@pytest.mark.parametrize("up", [2.0 ** 16, 2.0 ** 20, 2.0 ** 60])
@pytest.mark.parametrize("N,K", SHAPES)
@pytest.mark.parametrize("D,Dq,Dv,H", [(144, 128, 128, 16), (576, 512, 512, 16), (272, 256, 256, 32)])
def test_a_large_record_that_is_not_attended(up, N, K, D, Dq, Dv, H):
    """It scores far below the others, whatever its size."""
    rng = np.random.default_rng(K + H)
    x = rng.standard_normal((K, D))
    x[K // 3] = -np.abs(rng.standard_normal(D)) * up
    raw = ro.encode(exact_bf16(x), Dq)
    num = ro.decode(raw, D, Dq)
    table = np.stack([rng.permutation(K) for _ in range(N)]).astype(np.int32)
    q = exact_bf16(np.abs(rng.standard_normal((N, H, D))) + 0.1)
    out, lse = slot_table(raw, table, q, D, Dq, Dv, 0.03)
    hold(out, lse, num, table, q, Dv, 0.03, D)


@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("K", [128, 700, 4000])
def test_sizes_over_forty_binades(order, K):
    """Sizes that rise or fall along the row, scores that favour small records in some rows and large ones in others."""
    rng = np.random.default_rng(60 + K)
    D, Dq, Dv, H = 320, 256, 256, 20
    size = 2.0 ** np.linspace(-36, 4, K)[::order].round()
    x = rng.standard_normal((K, D)) * size[:, None]
    x[:, 128:256] *= 2.0 ** rng.integers(-9, 1, (K, 1))
    x[:, 256:] = rng.standard_normal((K, D - 256)) * 0.1
    x[:, 256] = np.linspace(-3, 3, K)                              # a number of the tail that orders the keys
    raw = ro.encode(exact_bf16(x), Dq)
    num = ro.decode(raw, D, Dq)
    table = np.arange(K, dtype=np.int32)[None]
    q = rng.standard_normal((1, H, D)) * 0.02
    q[0, :, 256] = np.linspace(-12, 12, H)
    q = exact_bf16(q)
    out, lse = slot_table(raw, table, q, D, Dq, Dv, 1.0)
    hold(out, lse, num, table, q, Dv, 1.0, D)


def test_scores_and_sizes_that_move_every_tile():
    """Records halve from tile to tile while some rows' scores rise and others stay: the references of a row and of its group
    move by small steps, many times."""
    rng = np.random.default_rng(61)
    D, K, H = 128, 128 * 60, 8
    size = 2.0 ** -(np.arange(K) // 128)
    x = rng.standard_normal((K, D)) * size[:, None]
    x[:, 0] = 4.0 * size
    raw = ro.encode(exact_bf16(x), 128)
    num = ro.decode(raw, D, 128)
    q = np.zeros((1, H, D))
    q[0, :, 0] = np.linspace(0.0, -8.0, H)                         # the small records score higher
    q = exact_bf16(q)
    for page in (1, 64):
        table = np.arange(K // page, dtype=np.int32)[None]
        out, lse = run_chunk(raw, table, np.array([K], dtype=np.int32), q, np.array([0, 1], dtype=np.int32), D, 128, 128, 1.0, page)
        hold(out, lse, num, np.arange(K)[None], q, 128, 1.0, D)


def test_one_token_alone_and_as_the_last_of_two():
    """The same token through both kernels: alone over codes, in a chunk of two over bf16."""
    rng = np.random.default_rng(62)
    D, Dq, Dv, H, page, K = 576, 512, 512, 16, 16, 333
    raw, num, table, cs, q, q_start = chunk_case(rng, [2], [K], H, D, Dq, page)
    at = table[0][np.arange(K) // page] * page + np.arange(K) % page
    x = rng.standard_normal((K, D)) * 1e-3
    x[[3, 100]] = 0
    x[200] = -np.abs(rng.standard_normal(D)) * 2.0 ** 14
    raw[at] = ro.encode(exact_bf16(x), Dq)
    num = ro.decode(raw, D, Dq)
    q = exact_bf16(np.abs(q) * 20)
    two, lse_two = run_chunk(raw, table, cs, q, q_start, D, Dq, Dv, 0.05, page)
    one, lse_one = run_chunk(raw, table, cs, q[1:2], np.array([0, 1], dtype=np.int32), D, Dq, Dv, 0.05, page)
    o, s, bo, bs = attended(num[at], q[1], Dv, 0.05, D)
    assert np.all(np.abs(numbers(one)[0] - o) <= bo) and np.all(np.abs(numbers(lse_one)[0] - s) <= bs)
    # (weights of 8 bits instead of 11 in the chunk)
    p = np.exp(0.05 * (q[1] @ num[at].T) - s[:, None])
    assert np.all(np.abs(numbers(two)[1] - numbers(one)[0]) <= 2 * bo + 2.0 ** -8 * (p @ np.abs(num[at][:, :Dv])))


def test_the_longest_context_of_single_tokens_over_codes():
    """131072 keys, the most that the kernel is given, with records of zeros and of several sizes among them."""
    rng = np.random.default_rng(63)
    D, K, H, page = 128, 131072, 4, 64
    x = (rng.standard_normal((K, D)) * 2.0 ** rng.integers(-14, -8, (K, 1))).astype(np.float32)
    x[rng.random(K) < 0.01] = 0
    x[:, 3] += 0.001
    fmt = hs.RecordFormat(D, 128)
    x = torch.from_numpy(x).to(DEV).to(torch.bfloat16)
    raw = hs.write_records(fmt, x, torch.zeros((K, fmt.entry_bytes), dtype=torch.uint8, device=DEV)).cpu().numpy()
    num = ro.decode(raw, D, 128)
    order = rng.permutation(K // page)
    moved = np.empty_like(raw).reshape(K // page, page, -1)
    moved[order] = raw.reshape(K // page, page, -1)
    q = exact_bf16(rng.standard_normal((1, H, D)) * 400)
    out, lse = run_chunk(moved.reshape(K, -1), order[None].astype(np.int32), np.array([K], dtype=np.int32), q,
                         np.array([0, 1], dtype=np.int32), D, 128, 128, 1.0, page)
    hold(out, lse, num, np.arange(K)[None], q, 128, 1.0, D)
