// Which tokens, chunks and runs a workgroup of the selective scan touches: plain arithmetic, in a header of its own so that it can be
// compiled and checked without a GPU.  Offsets of a packed batch are what a caller gives and nobody has looked at; whatever they are, and whichever
// sequence is taken for the one that holds a token, what comes out of here lies inside the tensors.
#pragma once

namespace hgrn2 {

constexpr int at_least(int v, int least) { return v < least ? least : v; }
constexpr int at_most(int v, int most) { return v > most ? most : v; }

// First token of the sequence that token t < hi belongs to, and the one behind its last, from what the offsets say (start, end in [0, T]; hi is the one
// behind the last token of all).  Offsets that rise say nothing else; others may name a sequence that t is not in, which is then made to hold it.
constexpr int place_first(int start, int t) { return at_most(start, t); }
constexpr int place_end(int end, int t, int hi) { return at_least(at_most(end, hi), t + 1); }

// ---- walks over the tokens [max(t0, lo), t1) of a run, not empty, in chunks of CT from t0 on ---------------------------
// The chunks of a walk: the first token of the first one, a multiple of CT behind t0, and how many.
struct SsmChunks { int first, count; };
constexpr SsmChunks ssm_chunks(int t0, int from, int t1, int CT)
{
    const int first = t0 + (from - t0) / CT * CT;
    return SsmChunks{first, (t1 - first + CT - 1) / CT};
}
// Forward, outputs: all chunks from t0 on, so that every state a chunk starts from is left.
constexpr SsmChunks ssm_chunks_forward(int t0, int t1, int CT) { return ssm_chunks(t0, t0, t1, CT); }
// Forward, from zero: nobody asks for what was before the sequence of the run's last token began, at `beg` < t1.
constexpr SsmChunks ssm_chunks_to_end(int t0, int t1, int beg, int CT) { return ssm_chunks(t0, at_least(beg, t0), t1, CT); }
// Reverse: down to the chunk that holds the run's first token of a sequence.  Of those before it there are no states: a forward run without
// such a token leaves them as they were, and runs of the two directions begin at different tokens.
constexpr SsmChunks ssm_chunks_back(int t0, int lo, int t1, int CT) { return ssm_chunks(t0, at_least(lo, t0), t1, CT); }
// Reverse, from zero: only the sequence of the run's first token reaches the runs before; it ends at `end` > max(t0, lo).
constexpr int ssm_end_back(int t1, int end) { return at_most(t1, end); }

// Tokens of the chunk at tc that may be read are tc + ssm_chunk_token(i, ...), i in [0, CT).
struct SsmTokens { int first, last; };
constexpr SsmTokens ssm_tokens_of(int tc, int t0, int lo, int t1, int CT) { return SsmTokens{at_least(at_least(t0, lo) - tc, 0), at_most(t1 - 1 - tc, CT - 1)}; }
constexpr int ssm_chunk_token(int i, SsmTokens in) { return at_most(at_least(i, in.first), in.last); }

// Packed: the run that the sequence of a run's first token begins in, from its first token, and the one that the sequence of its last token ends in.
constexpr int ssm_first_run(int beg, int run_len) { return beg / run_len; }
constexpr int ssm_last_run(int end, int run_len) { return (end - 1) / run_len; }

}   // namespace hgrn2
