// Launch planning of token_logprobs: host arithmetic only (no HIP, no allocation), so that it can also be compiled and
// exercised on a machine without a GPU.
#pragma once

#include "../../include/spdecode.h"

#include <stddef.h>
#include <stdint.h>

namespace spd {

// What a slice of a row leaves for the launch that joins them.
struct LogprobsPart {
    float m, r, z, s;
    int above, top;
};

namespace plan {

constexpr int kChunk = 8;  // logits whose maximum is kept

struct LogprobsPlan {
    int threads, stripes, slice, slices;  // of a workgroup, chunks of its threads at most, logits of a slice, slices of a row
};

constexpr int kMostSlice = 131072 - kChunk;  // (32 chunks for each of 512 threads, one of them for a start within 16 bytes)

inline LogprobsPlan make_logprobs_plan(int64_t rows, int64_t vocab)
{
    LogprobsPlan pl;
    // a workgroup a row, and slices where that leaves CUs idle
    int64_t slices = rows > 0 && rows <= 128 ? 256 / rows : 1;
    slices = slices < vocab / 16384 ? slices : vocab / 16384;
    const int64_t fit = (vocab + kMostSlice - 1) / kMostSlice;
    pl.slices = (int)(slices > fit ? slices : fit);
    pl.slice = (int)((vocab + pl.slices - 1) / pl.slices);
    pl.slice = (pl.slice + kChunk - 1) / kChunk * kChunk;  // (the bound is a multiple of a chunk)
    pl.threads = pl.slice <= 8192 ? 256 : 512;
    const int chunks = (pl.slice + 2 * kChunk - 2) / kChunk;  // (a slice that starts within 16 bytes has one more)
    pl.stripes = pl.threads == 256 ? (chunks <= 256 * 4 ? 4 : 8) : chunks <= 512 * 8 ? 8 : chunks <= 512 * 16 ? 16 : 32;
    return pl;
}

inline size_t logprobs_workspace(int64_t rows, int64_t vocab, int top)
{
    const LogprobsPlan pl = make_logprobs_plan(rows, vocab);
    return pl.slices > 1 ? (size_t)rows * pl.slices * (sizeof(LogprobsPart) + (size_t)top * 8) : 0;
}

// What no call of at most so many rows, logits and alternatives passes: few rows are cut into up to 256 slices in all, others as far as a slice holds.
inline size_t logprobs_workspace_of_any(int64_t rows, int64_t vocab, int top)
{
    const int64_t few = (rows < 128 ? rows : 128) * (vocab / 16384), fit = (vocab + kMostSlice - 1) / kMostSlice;
    const int64_t cut = vocab / 16384 > 1 ? (few < 256 ? few : 256) : 0, long_rows = fit > 1 ? rows * fit : 0;
    return (size_t)(cut > long_rows ? cut : long_rows) * (sizeof(LogprobsPart) + (size_t)top * 8);
}

}  // namespace plan
}  // namespace spd
