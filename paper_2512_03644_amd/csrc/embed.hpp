// Embedding of tokens with scaling, and its gradient by sorted tokens (embed.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ffsnap {

struct EmbedArgs {
    const uint8_t* rows;   // the table, or the gradient of the embedded tokens
    uint64_t rows_stride;  // elements
    const int64_t* ids;
    uint64_t n_tokens, vocab, width;
    float scale;
    uint8_t* out;  // the embedded tokens, or the table's gradient
    uint64_t out_stride;
};

uint64_t embed_workspace(uint64_t n_tokens, uint64_t vocab, uint64_t width);
hipError_t launch_embed(const EmbedArgs& a, uint32_t dtype, hipStream_t stream);
hipError_t launch_embed_grad(const EmbedArgs& a, uint32_t dtype, bool add, void* workspace, hipStream_t stream);

}  // namespace ffsnap
