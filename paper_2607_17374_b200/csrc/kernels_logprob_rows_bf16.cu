// Class log probabilities of short rows, bf16 (a file a type: they compile side by side).
#define LOGPROB_ROWS_TYPE 1
#include "logprob_rows.cuh"
