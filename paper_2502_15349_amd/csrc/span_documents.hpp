// Launch interface of the spans of packed documents.
#pragma once
#include "span.hpp"

namespace ae {

struct SpanDocuments {
  const int32_t* offsets;  // per batch entry n_docs + 1 offsets, `offset_stride` apart
  const int32_t* prefix;   // per batch entry n_docs lengths, `prefix_stride` apart; null: none
  int64_t offset_stride, prefix_stride;
  int B, L, n_docs, kind, window;
  int32_t *begin, *end;    // [B, L]
};
hipError_t launch_span_documents(const SpanDocuments& p, hipStream_t s);

}  // namespace ae
