// How a call of the vocabulary loss or of its gradient is cut up: sizes in, counts out, by the call's sizes and types alone.  Host code only.
#pragma once
#include <algorithm>
#include <cstdint>

namespace prsgd {

constexpr int kPairs = 74;                     // CTA pairs of the GPU (148 SMs)
constexpr int64_t kVtLongest = 8192;           // products that one running sum of the tensor cores takes in a gradient of 16-bit types

inline int64_t up(int64_t x, int64_t by) { return (x + by - 1) / by; }
inline int64_t up_to(int64_t x, int64_t by) { return up(x, by) * by; }

constexpr int64_t kLargestApart = 4096;        // fp16 gradients of more tokens: their largest |dloss| + |dlse| by a launch of its own (4 x 2100 x 512 x 128 40 us with it, 38 without; 4 x 8192 94 and 96; 16384 x 1000 x 256 130 and 139)

struct VocabCuts {
  int64_t Tp;                                  // rows of the copy of H
  int64_t tm;                                  // tiles along the tokens
  int tiles, td, kd;                           // tiles along the vocabulary, along D; blocks of 64 of D
  int64_t tasks;                               // at most
  int longest;                                 // gradient of 16-bit types: a contraction of more than kVtLongest products (of tokens or columns; dH's: 16384 at most)
  // loss
  int run, runs;                               // tiles along the vocabulary of a task, tasks of a group and 256 tokens
  // gradient
  int piece, pieces, gp;                       // columns of a piece of the vocabulary (a multiple of 256), pieces of a group, columns of a row of G
  int64_t seqs;                                // pieces of all groups
  int parts, kpart;                            // parts of dH's contraction, blocks of 64 of one
  int run_w;                                   // tiles of dW along the vocabulary of a task
  int h_first;                                 // of the uses of a piece: dH before dW
  int last_tiles, last_blocks;                 // tiles, blocks of 64 of a group's last piece
  int lag, slots;                              // uses follow G by that many pieces; pieces of G that have a place
};

// The loss of few tokens a group has its own form without tensor cores, where H fits in shared memory: two launches instead of three, but a class
// costs each token a sum over a warp.
// fp32, up to eight tokens: no copy of W as pairs (against the form of many tokens, us with cold caches; 1 x 32000 x 1024: one token 37 against 100, three 41 and 102, eight
// 55 and 101; 4 x 8 x 100000 x 256 211 and 318; 16 x 8 x 1000 x 1024 37 and 64; 64 x 4 x 5000 x 300 172 and 305).
// 16 bits, one or two tokens, while the tokens' classes are few (1 x 1 x 32000 x 1024 27 against 34, 1 x 2 31 and 35, 16 x 2 x 4000 x 1024 49 and 49; of more the sums decide:
// 1 x 2 x 100000 x 384 51 and 37, x 1024 68 and 64; 64 x 1 x 5000 x 300 170 and 162, 4 x 2 x 100000 x 256 90 and 64).
constexpr int kFewTokens = 8, kFewTurn = 4;    // tokens of a group at most, of a block at a time
constexpr int64_t kFewSmem = 96 * 1024;        // H of a block's tokens as fp32
constexpr int64_t kFewSums = 1 << 17;
inline bool vocab_few(bool fp32, int64_t groups, int64_t T, int64_t V, int D) {
  return T <= (fp32 ? kFewTokens : 2) && (T <= 2 ? T : kFewTurn) * up_to(D, 8) * 4 <= kFewSmem && (fp32 || groups * T * V <= kFewSums);
}

// The same for the gradient of a token or two: W is read and dW written once (against the form of many tokens, us with cold caches; 1 x 1 x 32000 x 1024 bf16 49 against 77,
// fp32 80 and 274; 1 x 131072 x 2048 bf16 270 and 351; 16 x 2 x 1000 x 1024 bf16 33 and 51; 64 x 1 x 5000 x 300 bf16 531 and 855.  Rows off 16 bytes, bf16: 1 x 1 x 32000 x 1024 157
// and 153, 1 x 2 149 and 153, 1 x 131072 x 2048 903 and 1095, 16 x 2 x 1000 x 1024 84 and 96, 4 x 2 x 100000 x 256 464 and 569).
constexpr int kFewGradTokens = 2, kFewGradDim = 2048;
inline bool vocab_few_grad(int64_t T, int D) { return T <= kFewGradTokens && D <= kFewGradDim; }

// split: fp32 operands, two planes each.
inline VocabCuts vocab_cuts(bool split, bool grad, int64_t groups, int64_t T, int64_t V, int D) {
  VocabCuts c{};
  const int planes = split ? 2 : 1;
  c.Tp = up_to(std::max<int64_t>(T, 1), 64);
  const int64_t tm = up(c.Tp, 256), nv = up(V, 256), td = up(D, 256);
  c.tm = tm; c.tiles = (int)nv; c.td = (int)td; c.kd = (int)up(D, 64);
  if (!grad) {
    // A run: tiles along the vocabulary whose maxima and sums one task keeps in registers; longer ones leave fewer parts behind, as long
    // as every pair gets eight.
    c.run = (int)std::max<int64_t>(1, std::min<int64_t>(8, groups * tm * nv / (8 * kPairs)));
    c.runs = (int)up(nv, c.run);
    c.tasks = groups * tm * c.runs;
    return c;
  }
  c.longest = !split && std::max<int64_t>(T, D) > kVtLongest;
  // A piece of G takes about 64 MB (8192 x 65536 x 2048: 16 MB 5.85 ms, 32 5.34, 64 5.04, 128 and 256 5.05: dH is added to once a piece).
  const int64_t fit = (64ll << 20) / (c.Tp * 2 * planes) / 256 * 256;
  c.piece = (int)std::min<int64_t>(nv * 256, std::max<int64_t>(512, fit));
  c.pieces = (int)up(V, c.piece);
  c.piece = (int)(up(nv, c.pieces) * 256);     // (equal ones)
  c.pieces = (int)up(V, c.piece);
  c.gp = (int)up_to(std::min<int64_t>(c.piece, V), 64);
  const int64_t npv = c.piece / 256;
  c.seqs = groups * c.pieces;
  // Parts of dH's contraction: one for every 4096 columns, and more while there are not two tiles a pair, but of 1024 or more.
  const int64_t few = up(2 * kPairs, tm * td);
  c.parts = (int)std::max<int64_t>(1, std::min<int64_t>(std::max<int64_t>(c.piece / 4096, std::min<int64_t>(few, c.piece / 1024)), 32));
  // Tiles of dW along the vocabulary that are one task: claiming takes about 2 us, as long as the products of 8 blocks of 64 tokens.
  c.run_w = (int)std::max<int64_t>(1, std::min<int64_t>(8 * 64 / std::min<int64_t>(c.Tp, 512), c.seqs * npv * td / (4 * kPairs)));
  c.kpart = (int)up(up(std::min<int64_t>(c.piece, V), 64), c.parts);
  c.h_first = c.kpart > c.Tp / 64 * c.run_w;   // the longer uses of a piece first
  c.last_tiles = (int)(nv - (c.pieces - 1) * npv);
  c.last_blocks = (int)up(V - (int64_t)(c.pieces - 1) * c.piece, 64);
  // Uses of a piece follow its tiles of G by as many pieces as hold two tiles a pair (16 groups of 64 tokens and 1000 classes: all G first); a
  // piece's place is taken again as many later.
  c.lag = (int)std::max<int64_t>(1, std::min<int64_t>(c.seqs, up(2 * kPairs, tm * npv)));
  c.slots = (int)std::min<int64_t>(c.seqs, 2 * c.lag + 1);
  c.tasks = c.seqs * (tm * npv + up(npv, c.run_w) * td + tm * td * c.parts);
  return c;
}

}  // namespace prsgd
