// Tokens drawn from rows of logits and drafted tokens verified: arguments, and the launches of draws.hip.
#pragma once

#include "logits.h"

namespace lb {

constexpr int64_t kMaxDrawVocab = 1 << 21;
constexpr int64_t kMaxDrafts = 128;

// A row's entries are summed in blocks of this many bytes, a wave's four loads, which begin on 16-byte boundaries of the logits.
// What is kept of a block, sum_j 2^((z_j - ref) c), tells where in the row a running sum is passed; the one block is then read again.
constexpr int kBlockBytes = 4096;
struct BlockSum {
    float ref, sum;
};
// blocks of a row, at most (the first may begin before the row does)
inline int64_t blocks_of(int64_t vocab, int size) { return (vocab * size + (16 - size) + kBlockBytes - 1) / kBlockBytes; }

// Rows of logits: `each` of them for a request.
struct RowSet {
    const void* z;
    int64_t ld, ld_request;
    int each;
};

struct DrawArgs {
    const void* z;
    int64_t rows, ld;
    int vocab;
    double s;                // 1 / temperature
    Factor c;
    const float* uniform;
    int64_t* tokens;
    float* logp;
};

struct VerifyArgs {
    RowSet target, draft;    // draft.z null: q is 1 at the drafted token
    int64_t requests;
    int drafts, vocab;
    double s, draft_s;
    Factor c, draft_c;
    const float* draft_logp; // null: from draft.z
    const int64_t *drafted, *lengths;
    const float *uniform, *last_uniform;
    int64_t *tokens, *count;
    float* logp;
};

// What is drawn from where a position's token is not accepted.
enum { kFromTarget = 0, kWithout = 1, kRest = 2 };     // p; p without the token; max(p - q, 0)
struct Exponent {            // of 2, in two parts, the second times ln 2
    float high, low;
};
struct Position {
    double sum;              // p_j = 2^((z_j - top) c) / sum
    float top;
    Exponent p;              //     = 2^((z_j - top) c + p)
    float q_ref;
    Exponent q;              // q_j = 2^((zq_j - q_ref) cq + q)
    int accepted, mode, x;   // x: the drafted token
    float logp;              // its log-probability
};
struct Asked {
    int x, inside;           // the drafted token; it lies in the vocabulary
    float u, given, z, zq;   // given: draft_logp; z, zq: its logits
};

// where the parts of a call's workspace are, in bytes behind the blocks' sums of the target's rows (draws.hip); whole: how much there is of it
struct VerifySpace {
    size_t draft, rest, asked, tickets, whole;
};
// drafter: its rows are there; both: they are summed as well
VerifySpace verify_space(int64_t requests, int64_t drafts, int64_t vocab, int size, bool drafter, bool both);
size_t draw_space(int64_t rows, int64_t vocab, int size);

hipError_t launch_draw(const DrawArgs& a, int dtype, void* ws, hipStream_t st);
hipError_t launch_verify(const VerifyArgs& a, int dtype, void* ws, hipStream_t st);

}  // namespace lb
