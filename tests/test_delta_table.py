"""The table of chunks for offsets that fall, of many documents: their chunks together are more than 32 bits hold and than the table has room for.
Every row stays inside of the table and of the tokens."""
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2507_10392_amd as zs
from paper_2507_10392_amd import build

gpu = pytest.mark.gpu

# (T, documents, the offsets' pattern): documents of T tokens and empty ones in turn, of all tokens but for a few, and offsets anywhere.
SIZES = [(1 << 26, 4400, "0T"), (1 << 26, 8192, "0T"), (1 << 26, 1 << 18, "0T"), (1500000, 1 << 18, "0T"), (1 << 21, 1 << 18, "0T"), (1 << 26, 1 << 18, "any"),
         (1 << 26, 1023, "0T"), (1 << 26, 1025, "steps"), (64, 1 << 18, "0T"), (1, 1 << 18, "0T")]


def offsets_of(T, n, pattern):
    if pattern == "0T":
        return np.where(np.arange(n + 1) % 2, T, 0).astype(np.int32)
    if pattern == "steps":
        return np.where(np.arange(n + 1) % 2, T - np.arange(n + 1) % 130, np.arange(n + 1) % 70).astype(np.int32)
    return np.random.default_rng(n).integers(-2 ** 31, 2 ** 31 - 1, n + 1, dtype=np.int64).astype(np.int32)


def room_of(T, n):
    return zs.delta_chunks_ints(T, n) // 4 - 1 - n


def expected(T, offsets):
    """Documents clipped to the tokens, and to the chunks that are left, in whole numbers without a limit -> first token, tokens, first chunk."""
    n, room = len(offsets) - 1, room_of(T, len(offsets) - 1)
    at = np.clip(offsets.astype(np.int64), 0, T)
    first, count = at[:-1], np.maximum(at[1:] - at[:-1], 0)
    chunks = -(-count // 64)
    chunk0 = np.minimum(np.concatenate(([0], np.cumsum(chunks)[:-1])), room)
    return first, np.minimum(count, (room - chunk0) * 64), chunk0


# The kernel's turns with its own functions and 32-bit sums, which are looked at as they are formed.
PROGRAM = r"""
#include "kernels.h"
#include <algorithm>
#include <cstdio>
#include <vector>
using namespace zs;
static bool wrapped = false;
static int sum(int a, int b) {
  int c;
  wrapped |= __builtin_add_overflow(a, b, &c);
  return c;
}
int main() {
  int T, n, nchunks;
  while (scanf("%d %d %d", &T, &n, &nchunks) == 3) {
    std::vector<int> offsets(n + 1);
    for (int& x : offsets)
      if (scanf("%d", &x) != 1) return 1;
    int before = 0;
    for (int d0 = 0; d0 < n; d0 += DELTA_TURN) {
      int turn = 0;
      for (int d = d0; d < std::min(n, d0 + DELTA_TURN); ++d) {
        const int first = std::min(std::max(offsets[d], 0), T), count = std::max(std::min(std::max(offsets[d + 1], 0), T) - first, 0);
        wrapped |= (long long)before + turn > 0x7fffffff;
        const DeltaPlace at = delta_place(before, turn, count, nchunks);
        printf("%d %d\n", at.chunk0, at.tokens);
        turn = sum(turn, delta_chunks_of(count));
      }
      wrapped |= (long long)before + turn > 0x7fffffff;
      before = delta_turn_end(before, turn, nchunks);
    }
    printf("%d %d\n", before, (int)wrapped);
  }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = tmp_path_factory.mktemp("table")
    src, exe = out / "table.hip", out / "table"
    src.write_text(PROGRAM)
    subprocess.run([build._hipcc(), *build.FLAGS, "-w", "-I", build.CSRC, str(src), "-o", str(exe)], check=True, capture_output=True)
    return exe


@pytest.mark.parametrize("T,n,pattern", SIZES)
def test_places_stay_inside_of_the_table(program, T, n, pattern):
    offsets, room = offsets_of(T, n, pattern), room_of(T, n)
    text = "%d %d %d\n%s\n" % (T, n, room, " ".join(map(str, offsets)))
    out = subprocess.run([str(program)], check=True, capture_output=True, text=True, input=text, env=dict(os.environ, HIP_VISIBLE_DEVICES="-1")).stdout
    got = np.array(out.split(), dtype=np.int64).reshape(-1, 2)
    assert got.shape[0] == n + 1 and got[n, 1] == 0, "a sum of 32 bits wrapped"
    chunk0, tokens = got[:n].T
    assert (chunk0 >= 0).all() and (tokens >= 0).all() and (chunk0 + -(-tokens // 64) <= room).all() and 0 <= got[n, 0] <= room
    first, want_tokens, want_chunk0 = expected(T, offsets)
    assert np.array_equal(tokens, want_tokens) and np.array_equal(chunk0, want_chunk0) and (first + tokens <= T).all()


@gpu
@pytest.mark.parametrize("T,n,pattern", SIZES)
def test_table_of_offsets_that_fall(gpu_device, T, n, pattern):
    print("[case] falling offsets", T, n, pattern, flush=True)
    offsets, ints, beside = offsets_of(T, n, pattern), zs.delta_chunks_ints(T, n), 1 << 16
    buf = torch.full((ints + 2 * beside,), -7, dtype=torch.int32, device="cuda")
    zs.ops.delta_chunks(torch.cuda.current_stream().cuda_stream, T, n, torch.from_numpy(offsets).cuda(), buf[beside:beside + ints])
    t = buf.cpu().numpy()
    assert (t[:beside] == -7).all() and (t[beside + ints:] == -7).all()
    t = t[beside:beside + ints].reshape(-1, 4).astype(np.int64)
    docs, chunks = t[1:1 + n], t[1 + n:]
    docs = docs[np.argsort(docs[:, 3], kind="stable")]
    first, tokens, chunk0 = expected(T, offsets)
    assert np.array_equal(docs, np.stack((first, tokens, chunk0, np.arange(n)), 1))
    many = -(-tokens // 64)
    d = np.repeat(np.arange(n), many)
    i = np.arange(len(d)) - np.repeat(np.cumsum(many) - many, many)
    assert np.array_equal(chunks[:len(d)], np.stack((first[d] + 64 * i, np.minimum(tokens[d] - 64 * i, 64), d, i), 1))
    assert (chunks[len(d):] == 0).all()
